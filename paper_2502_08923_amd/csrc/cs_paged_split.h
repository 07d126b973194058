// How the work of an attention over pages is cut: which query rows and tokens a workgroup has, found on
// the device from the lengths, and what several workgroups have of a row, joined by a merge.
#pragma once

#include "cs_paged.h"

struct pa_args {
    const void* q;
    int64_t q_row, q_head;
    void* out;
    int64_t out_row, out_head;
    int H, G, window;
    float scale2;             // scale * log2(e): scores in base-2 units
};

// ---- which query rows and tokens a workgroup has --------------------------------------------------
// The G * rows query rows of a stream's KV head (row n: block row n / G, head n % G of the group) are
// cut into tiles of TR. Streams with qr_lo < G * rows <= qr_hi take part in a launch.  The tokens of a
// tile are cut into ranges of `chunk`, where that fills the chip better; lengths are only known on the
// device, so the cut is made there, by every workgroup for itself: each lane prices another number of
// ranges for the longest stream (rounds of the chip that all ranges of all streams then take, a round
// costing its tokens and, in the same unit, a workgroup's start and end), and the cheapest is taken of
// those that there is room for.  Room is what the host's cut needs, which takes every stream to be as
// long as the longest, or one round of the chip: where single tiles of all streams fill the chip by
// that count (32 streams of 8 KV heads), a long one among short ones is not cut finer.  A batch of more
// than 64 streams takes the host's cut itself, whatever its lengths are, and where it has row offsets
// every workgroup walks them 64 at a time until its own: that is for hundreds of streams (single tokens
// behind 100, 8 heads of 128 a KV head: 256 streams 9.2 us against 7.8 without offsets, 1024 38 against
// 17, 4096 353 against 52).  (Against the host's cut for all: 2048 rows and 15 single tokens behind 4 to
// 16 thousand 740 -> 685 us, two ragged float32 prompt blocks 185 -> 152 us, eight equal streams 120 ->
// 122 us.)
struct pa_tile {
    int b, n0, QR;            // stream, first query row, query rows of the stream
    int row0, rows, L;        // its first row, rows, length
};
struct pa_plan {
    int TR, qr_lo, qr_hi;
    int slots, start, join;   // workgroups that run at once; tokens' worth of a workgroup's ends, and of the merge
    int n_max, step;          // most ranges; distance of the numbers priced
    int chunk;                // the host's cut
    int entries;              // (tile, range) pairs that there is room for
    float* po;                // [entry][KVH][TR][hd] partial outputs
    float2* pml;              // [entry][KVH][TR] their (maximum, sum)
    int4* who;                // [entry] (first row, first query row, query rows, range | ranges << 16) for the merge; ranges 0: nobody
};
struct pa_work {
    pa_tile T;
    int entry;                // this (tile, range) among all; the ranges of a tile follow each other
    int split, nsplit, chunk; // range, ranges of the stream's tiles, tokens of one (the last takes what is left)
};

// tiles of stream b, and the tokens that one of them walks
__device__ __forceinline__ int2 pa_extent(const cs_pages_dev& D, int G, int window, const pa_plan& P, int b) {
    const int rows = cs_stream_rows(D, b).y;
    const int64_t qr = (int64_t)rows * G;
    if (qr <= P.qr_lo || qr > P.qr_hi) return make_int2(0, 0);
    int span = min(cs_stream_len(D, b) + rows, D.cap);
    if (window) span = (int)min((int64_t)span, (int64_t)window + min(rows, P.TR / G + 1) + 32);
    return make_int2((int)((qr + P.TR - 1) / P.TR), max(span, 1));
}
// Reductions over the wave in registers (data-parallel primitives: rows of 16, then row ends to the
// rows behind them); a lane that a step does not reach combines with `id`.  Lane 63 has everything.
template <typename F>
__device__ __forceinline__ int pa_wave_reduce(int v, int id, F f) {
#define PA_DPP(ctrl, rows) v = f(v, __builtin_amdgcn_update_dpp(id, v, ctrl, rows, 0xf, false))
    PA_DPP(0x111, 0xf);
    PA_DPP(0x112, 0xf);
    PA_DPP(0x114, 0xf);
    PA_DPP(0x118, 0xf);
    PA_DPP(0x142, 0xa);
    PA_DPP(0x143, 0xc);
#undef PA_DPP
    return v;
}
__device__ __forceinline__ int pa_wave_scan(int v) {                       // inclusive
    return pa_wave_reduce(v, 0, [](int a, int b) { return a + b; });
}

__device__ __forceinline__ bool pa_find_entry(const cs_pages_dev& D, int G, int window, const pa_plan& P, int wg, pa_work& o) {
    const int lane = threadIdx.x & 63, B = D.p.batch;
    int chunk = P.chunk, b = -1, at = 0, n_b = 1;
    if (B <= 64) {            // (a wave has a lane for each stream)
        const int2 e = lane < B ? pa_extent(D, G, window, P, lane) : make_int2(0, 0);
        if (P.n_max > 1) {
            const int longest = __builtin_amdgcn_readlane(pa_wave_reduce(e.y, 0, [](int a, int b) { return max(a, b); }), 63);
            const int n = 1 + lane * P.step;
            const int cut = max(((longest + n - 1) / n + 31) & ~31, 32);
            const float inv = 1.0f / (float)cut;
            int count = 0;
            for (int i = 0; i < B; ++i) {
                const int tokens = __builtin_amdgcn_readlane(e.y, i), q = (int)((float)tokens * inv), r = tokens - q * cut;
                count += __builtin_amdgcn_readlane(e.x, i) * (q + (r > 0) + (r > cut));       // (q is off by one at most)
            }
            float cost = ceilf((float)count * (float)D.p.n_kv_heads / (float)P.slots) * (float)(cut + P.start) + (n > 1 ? (float)(P.join + n) : 0.f);
            if (n > 1 && (n > P.n_max || cut < 64 || count > P.entries)) cost = INFINITY;
            // (costs are positive: their bits are ordered as they are)
            const int best = __builtin_amdgcn_readlane(pa_wave_reduce(__float_as_int(cost), 0x7f800000, [](int a, int b) { return min(a, b); }), 63);
            chunk = __builtin_amdgcn_readlane(cut, __ffsll(__ballot(__float_as_int(cost) == best)) - 1);
        }
        int n = e.x ? min(P.n_max, max(1, (e.y + chunk - 1) / chunk)) : 1, mine = e.x * n, incl = pa_wave_scan(mine);
        if (__builtin_amdgcn_readlane(incl, 63) > P.entries) {   // (row offsets that make no sense: more tiles than rows allow)
            n = 1;
            mine = e.x;
            incl = pa_wave_scan(mine);
        }
        const int total = min(__builtin_amdgcn_readlane(incl, 63), P.entries);
        if (wg >= total) return false;
        const int idx = total - 1 - wg;                     // the last tiles of a prompt see most: they go first
        const int l = __ffsll(__ballot(incl > idx)) - 1;
        b = l;
        n_b = __builtin_amdgcn_readlane(n, l);
        at = idx - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(mine, l));
        o.entry = idx;
    } else if (!D.row0 && P.n_max == 1) {                    // equal shares, whole contexts: nothing to look up
        const int tiles = pa_extent(D, G, window, P, 0).x;
        if (wg >= B * tiles) return false;
        b = wg / tiles;
        at = wg - b * tiles;
        o.entry = wg;
    } else {
        int base = 0;
        for (int b0 = 0; b0 < B; b0 += 64) {
            const int2 e = b0 + lane < B ? pa_extent(D, G, window, P, b0 + lane) : make_int2(0, 0);
            const int n = e.x ? min(P.n_max, max(1, (e.y + chunk - 1) / chunk)) : 1;
            const int mine = e.x * n, incl = pa_wave_scan(mine);
            const unsigned long long past = __ballot(base + incl > wg);
            if (past) {
                const int l = __ffsll(past) - 1;
                b = b0 + l;
                n_b = __builtin_amdgcn_readlane(n, l);
                at = wg - base - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(mine, l));
                break;
            }
            base += __builtin_amdgcn_readlane(incl, 63);
        }
        if (b < 0 || wg - at % n_b + n_b > P.entries) return false;       // (the second: as above)
        o.entry = wg;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    at = __builtin_amdgcn_readfirstlane(at);
    n_b = __builtin_amdgcn_readfirstlane(n_b);
    const int2 sr = cs_stream_rows(D, b);
    o.T.b = b;
    o.T.row0 = __builtin_amdgcn_readfirstlane(sr.x);
    o.T.rows = __builtin_amdgcn_readfirstlane(sr.y);
    o.T.QR = o.T.rows * G;
    o.T.n0 = at / n_b * P.TR;
    o.T.L = __builtin_amdgcn_readfirstlane(cs_stream_len(D, b));
    o.split = at % n_b;
    o.nsplit = n_b;
    o.chunk = __builtin_amdgcn_readfirstlane(chunk);
    return true;
}

// the same, noted down for the merge
__device__ __forceinline__ bool pa_find(const cs_pages_dev& D, int G, int window, const pa_plan& P, int wg, int kvh, pa_work& o) {
    const bool work = pa_find_entry(D, G, window, P, wg, o);
    if (P.n_max > 1 && kvh == 0 && threadIdx.x == 0)
        P.who[work ? o.entry : wg] = work ? make_int4(o.T.row0, o.T.n0, o.T.QR, o.split | o.nsplit << 16) : make_int4(0, 0, 0, 0);
    return work;
}

__device__ __forceinline__ void pa_store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void pa_store4(bf16_t* p, f32x4 v) {
    *reinterpret_cast<bf16x4*>(p) = (bf16x4){(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
}

// How a call is cut: the same for the workspace and the launches.
struct pa_part {
    int nt, TR, qr_lo, qr_hi, tiles;          // tiles: an upper bound; 0: no launch
    int slots, start, join, n_max, step, chunk, entries;
};
// fills what follows `tiles` for a launch over contexts of up to `len` tokens; returns the bytes of its workspace
int64_t pa_ranges(pa_part& t, int64_t len, int B, int KVH, int hd, int slots, int start, int join);
pa_plan pa_plan_of(const pa_part& t, char* ws, int KVH, int hd);
// joins the ranges of the launch before it, of the same grid; the outputs are of type D.p.dtype
int pm_launch(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s);
