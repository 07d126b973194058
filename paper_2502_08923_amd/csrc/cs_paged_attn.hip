// Attention of a chunk of new rows per stream over the pages of its cache (Sec. 3.2: the draft is
// appended to the context and evaluated in one pass; App. B.2: per-layer K, V).
//
//   out[r][h] = sum_t p_t v[t] / sum_t p_t,   p_t = exp(scale * q[r][h] . k[t] - max),   t <= L_b + i, t > L_b + i - window
//
// One pass over the tokens with the running maximum and sum of the softmax in float32.  Three kernels:
// bfloat16 caches with few query rows per KV head (the stream of keys and values is the bound) and with
// many (the multiplies are), float32 caches; and the merge of what several workgroups have of a row.
// They multiply with the matrix instructions, K as the A operand, so a lane (c, g) = (lane % 16, lane /
// 16) has four consecutive tokens of query row c in the result, which is what the second product wants
// of its B operand. No wave, workgroup or launch order enters a result: every sum has one order, given
// by the cut.
#include <algorithm>
#include <cmath>
#include <type_traits>

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

// The (max, sum, O) triples of W waves side by side in LDS -> the tile's rows: the output itself where
// the tokens are in one range, else this range's partial result.
template <int W, int HD, int ROWS, typename T_>
__device__ __forceinline__ void pa_finish(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, const pa_work& K, int kvh, int n_rows,
                                          const float* s_o, const float2* s_ml, int tid, int n_threads) {
    const pa_tile& T = K.T;
    constexpr int OROW = HD + 4;
    const int hd = D.p.head_dim;
#pragma unroll 1
    for (int idx = tid; idx < n_rows * (HD / 4); idx += n_threads) {
        const int n = idx / (HD / 4), d = idx % (HD / 4) * 4;
        float2 ml[W];
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            ml[w] = s_ml[w * ROWS + n];
            M = fmaxf(M, ml[w].x);
        }
        const float Ms = M == -INFINITY ? 0.f : M;
        f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[w].x - Ms);
            o += f * *reinterpret_cast<const f32x4*>(&s_o[(w * ROWS + n) * OROW + d]);
            l += f * ml[w].y;
        }
        const int i = (T.n0 + n) / A.G, h = kvh * A.G + T.n0 + n - i * A.G;
        const int64_t r = T.row0 + i;
        if (K.nsplit == 1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;           // a row that sees nothing: 0
            if (d < hd) pa_store4((T_*)A.out + r * A.out_row + h * A.out_head + d, o * inv);
            continue;
        }
        const int64_t at = ((int64_t)K.entry * D.p.n_kv_heads + kvh) * P.TR + n;
        if (d < hd) *reinterpret_cast<f32x4*>(P.po + at * hd + d) = o;
        if (d == 0) P.pml[at] = make_float2(M, l);
    }
}

// ---- few query rows: the stream of keys and values is the bound ---------------------------------
// Four waves share a tile of up to 48 query rows and take the 32-token blocks of a token range in turn;
// keys, values, scores and outputs stay in registers:
//   S^T[token][row] = K . Q^T           A = 16 key rows (a lane: 8 features of one), B = query rows
//   O^T[feature][row] += V^T . P^T      A = 16 features of 32 tokens, B = the probabilities as S^T left them
// The k index of the second product may run over the block's tokens in any order that both operands
// share, so lane (c, g) takes the tokens 4g..4g+3 of either 16-token half, which are the rows of S^T it
// holds already.  A lane loads 16 bytes of those eight value rows (8 features of each) and turns the 8
// x 8 square with 32 byte permutes into eight A fragments: fragment u has feature 8c + u in row c.  So
// the values lie in the pages as they come, and a wave's load takes whole rows. A page holds whole
// 16-token halves, so every load has one page and a uniform base: a buffer whose size ends with the
// last token.  Loads past it, and of pages that do not exist, return zeros and cost no traffic, and
// none sits behind a branch. Two blocks of keys and two of values per wave are in flight (32 KB a wave
// at head_dim 128); what bounds it then is memory: 8 streams of 11 rows behind 18431 tokens, head_dim
// 128, 4 heads a group, 606 MB: 109 to 115 us = 5.3 to 5.6 TB/s; 64 single tokens behind 2 to 8
// thousand, pages of 16 tokens, 1357 MB: 259 to 266 us = 5.1 to 5.2 TB/s; one stream of 16000: 22 us
// with the merge. Workgroups: one per compute unit (twice as many cost 7 %, four times 20 %: their
// starts, their ends and the merge).
#define PN_WAVES 4
template <int HD>
struct pn_kbuf { bf16x8 k[2][HD / 32]; };
template <int HD>
struct pn_vbuf { unsigned v[8][HD / 32]; };     // [row j][dword]: row 4g + j % 4 of half j / 4

template <int HD, int NT>
__global__ __launch_bounds__(64 * PN_WAVES) void k_paged_narrow(cs_pages_dev D, pa_args A, pa_plan P) {
    constexpr int KS = HD / 32, MT = HD / 16, VD = HD / 32;
    constexpr int VW = HD == 64 ? 2 : 4;                // dwords of one value load
    constexpr int VL = VD / VW;                         // loads per value row
    constexpr int VF = 2 * VW;                          // features of one value load
    constexpr int ROWS = 16 * NT, OROW = HD + 4, QROW = HD * 2 + 16;
    constexpr int MERGE_BYTES = PN_WAVES * ROWS * (OROW * 4 + 8), Q_BYTES = ROWS * QROW;
    __shared__ __attribute__((aligned(16))) unsigned char smem[MERGE_BYTES > Q_BYTES ? MERGE_BYTES : Q_BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const unsigned wg = cs_paged_wg();
    const int KVH = D.p.n_kv_heads, kvh = wg % KVH;
    pa_work K;
    if (!pa_find(D, A.G, A.window, P, wg / KVH, kvh, K)) return;
    const pa_tile& T = K.T;
    const int hd = D.p.head_dim;
    const int n_rows = min(ROWS, T.QR - T.n0);          // live query rows of the tile
    const int i_lo = T.n0 / A.G, i_hi = (T.n0 + n_rows - 1) / A.G;
    const int n_tok = min(T.L + i_hi + 1, D.cap);       // tokens that the tile's last row sees
    const int base = A.window ? max(0, T.L + i_lo - A.window + 1) & ~31 : 0;
    const int w_begin = (int)min((int64_t)base + (int64_t)K.split * K.chunk, (int64_t)n_tok);
    const int t_end = K.split == K.nsplit - 1 ? n_tok : (int)min((int64_t)w_begin + K.chunk, (int64_t)n_tok);
    // blocks between these need no mask
    const int open_lo = A.window ? T.L + i_hi - A.window + 1 : 0, open_hi = min(T.L + i_lo + 1, D.cap);
    const int w_first = A.window ? T.L + i_lo - A.window + 1 : 0;       // tokens before it are seen by no row of the tile

    // query rows into LDS
    for (int idx = tid; idx < ROWS * (HD / 8); idx += 64 * PN_WAVES) {
        const int n = idx / (HD / 8), seg = idx % (HD / 8);
        bf16x8 v = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
        if (n < n_rows && seg * 8 < hd) {
            const int i = (T.n0 + n) / A.G, h = kvh * A.G + T.n0 + n - i * A.G;
            v = *reinterpret_cast<const bf16x8*>((const bf16_t*)A.q + (T.row0 + i) * A.q_row + h * A.q_head + seg * 8);
        }
        *reinterpret_cast<bf16x8*>(smem + n * QROW + seg * 16) = v;
    }
    int q_last[NT], q_first[NT];                        // tokens that the lane's query rows see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = nt * 16 + c, i = (T.n0 + n) / A.G;
        q_last[nt] = n < n_rows ? T.L + i : -1;
        q_first[nt] = A.window ? T.L + i - A.window + 1 : 0;
    }

    const bf16_t* Kh = (const bf16_t*)D.p.k + kvh * D.p.k_head;
    const bf16_t* Vh = (const bf16_t*)D.p.v + kvh * D.p.v_head;
    const int32_t* tab = D.p.table + T.b * D.p.table_stride;
    constexpr unsigned NOWHERE = 0x80000000u;
    const unsigned kts = (unsigned)D.p.k_token * 2, vts = (unsigned)D.p.v_token * 2;      // bytes per token
    unsigned koff[KS], voff[4][VL];
#pragma unroll
    for (int s = 0; s < KS; ++s) koff[s] = s * 32 + g * 8 < hd ? c * kts + s * 64 + g * 16 : NOWHERE;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < VL; ++x) voff[j][x] = x * 16 * VF + c * VF < hd ? (4 * g + j) * vts + (x * 16 + c) * VF * 2 : NOWHERE;

    f32x4 oacc[MT][NT], lacc[NT];
    float m_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = -INFINITY;
        lacc[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const bf16_t one = (bf16_t)1.0f;
    const bf16x8 ones = (bf16x8){one, one, one, one, one, one, one, one};
    const float scale2 = A.scale2;
    __syncthreads();

    constexpr int STEP = 32 * PN_WAVES;
    // a lane holds the pages of one of the wave's next 64 blocks
    for (int seg0 = w_begin; seg0 < t_end; seg0 += 64 * STEP) {
        const int t_begin = seg0 + 32 * wave;
        const int n_all = t_begin < t_end ? min(64, (t_end - t_begin + STEP - 1) / STEP) : 0;
        int page0 = -1, page1 = -1;
        {
            const int64_t tb = (int64_t)t_begin + (int64_t)lane * STEP;
            if (tb < t_end) {
                page0 = tab[tb >> D.page_log2];
                const int e1 = (int)((tb + 16) >> D.page_log2);
                page1 = e1 < D.p.table_pages ? tab[e1] : -1;
            }
            page0 = (unsigned)page0 < (unsigned)D.p.n_pages ? page0 : -1;
            page1 = (unsigned)page1 < (unsigned)D.p.n_pages ? page1 : -1;
        }
        auto at = [&](int i) { return t_begin + i * STEP; };
        auto page_of = [&](int i, int a) { return __builtin_amdgcn_readlane(a ? page1 : page0, i); };
        auto buffer = [&](const bf16_t* head, int64_t page_stride, unsigned ts, int i, int a) {
            const int t = at(i) + 16 * a, page = i < n_all ? page_of(i, a) : -1;
            const int live = min(16, n_tok - t);
            const unsigned bytes = page >= 0 && live > 0 ? (live - 1) * ts + hd * 2 : 0;
            const char* p = (const char*)(head + (page >= 0 ? page : 0) * page_stride) + (int64_t)(t & (D.p.page_size - 1)) * ts;
            return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, CS_BUFFER_WORD3);
        };
        auto ldk = [&](pn_kbuf<HD>& buf, int i) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const auto rs = buffer(Kh, D.p.k_page, kts, i, a);
#pragma unroll
                for (int s = 0; s < KS; ++s) buf.k[a][s] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, koff[s], 0, 0));
            }
        };
        auto ldv = [&](pn_vbuf<HD>& buf, int i) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const auto rs = buffer(Vh, D.p.v_page, vts, i, a);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 0; x < VL; ++x) {
                        if constexpr (VW == 4) {
                            const auto t = __builtin_amdgcn_raw_buffer_load_b128(rs, voff[j][x], 0, 0);
#pragma unroll
                            for (int d = 0; d < 4; ++d) buf.v[4 * a + j][x * 4 + d] = t[d];
                        } else {
                            const auto t = __builtin_amdgcn_raw_buffer_load_b64(rs, voff[j][x], 0, 0);
#pragma unroll
                            for (int d = 0; d < 2; ++d) buf.v[4 * a + j][x * 2 + d] = t[d];
                        }
                    }
            }
        };
        auto block = [&](pn_kbuf<HD>& kb, pn_vbuf<HD>& vb, int i) {
            f32x4 sacc[2][NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                f32x4 z0 = (f32x4){0.f, 0.f, 0.f, 0.f}, z1 = z0;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const bf16x8 qb = *reinterpret_cast<const bf16x8*>(smem + (nt * 16 + c) * QROW + s * 64 + g * 16);
                    z0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb.k[0][s], qb, z0, 0, 0, 0);
                    z1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb.k[1][s], qb, z1, 0, 0, 0);
                }
                sacc[0][nt] = z0;
                sacc[1][nt] = z1;
            }
            __builtin_amdgcn_sched_barrier(0);
            ldk(kb, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = at(i), p0 = page_of(i, 0), p1 = page_of(i, 1);
            if (t0 < open_lo || t0 + 32 > open_hi || p0 < 0 || p1 < 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int t = t0 + 16 * a + 4 * g + j;
                            const bool sees = t <= q_last[nt] && t >= q_first[nt] && t < D.cap && (a ? p1 : p0) >= 0;
                            sacc[a][nt][j] = sees ? sacc[a][nt][j] : -INFINITY;
                        }
                if (t0 < w_first) {                     // (what has left every window may be anything, and 0 * anything must stay 0)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool gone = t0 + 16 * (j >> 2) + 4 * g + (j & 3) < w_first;
#pragma unroll
                        for (int d = 0; d < VD; ++d) vb.v[j][d] = gone ? 0u : vb.v[j][d];
                    }
                }
            }
            bool moved = false;
            float alpha[NT];
            bf16x8 pb[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float sv[8];
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sv[4 * a + j] = sacc[a][nt][j];
                float mx = fmaxf(fmaxf(sv[0], sv[1]), sv[2]);
                mx = fmaxf(fmaxf(mx, sv[3]), sv[4]);
                mx = fmaxf(fmaxf(mx, sv[5]), fmaxf(sv[6], sv[7]));
                mx = fa_row4_max(mx) * scale2;
                // the reference maximum follows the true one only when it is left behind by 2^8:
                // probabilities stay below 256, O and the row sum stay consistent, and O is rescaled a
                // handful of times per wave
                const bool up = mx > m_run[nt] + FA_RESCALE_LOG2;
                const float m_new = up ? mx : m_run[nt];
                const float m_safe = m_new == -INFINITY ? 0.f : m_new;
                alpha[nt] = up ? __builtin_amdgcn_exp2f(m_run[nt] - m_safe) : 1.0f;
                moved |= up;
                m_run[nt] = m_new;
                // rounded to bfloat16, the type of V in the product; the row sum is that of the rounded
                // values
#pragma unroll
                for (int j = 0; j < 8; ++j) pb[nt][j] = (bf16_t)__builtin_amdgcn_exp2f(fmaf(sv[j], scale2, -m_safe));
            }
            if (__any(moved)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    asm volatile("" : "+a"(lacc[nt]));
                    lacc[nt] *= alpha[nt];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        asm volatile("" : "+a"(oacc[mt][nt]));
                        oacc[mt][nt] *= alpha[nt];
                    }
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) lacc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[nt], lacc[nt], 0, 0, 0);
#pragma unroll
            for (int d = 0; d < VD; ++d) {
                // dword d of the eight rows: features 2d and 2d + 1 of the lane's
                unsigned lo[4], hi[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    lo[r] = __builtin_amdgcn_perm(vb.v[2 * r + 1][d], vb.v[2 * r][d], 0x05040100u);
                    hi[r] = __builtin_amdgcn_perm(vb.v[2 * r + 1][d], vb.v[2 * r][d], 0x07060302u);
                }
                typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
                const bf16x8 fl = __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], lo[2], lo[3]});
                const bf16x8 fh = __builtin_bit_cast(bf16x8, (u32x4){hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    oacc[2 * d][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fl, pb[nt], oacc[2 * d][nt], 0, 0, 0);
                    oacc[2 * d + 1][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh, pb[nt], oacc[2 * d + 1][nt], 0, 0, 0);
                }
            }
            // accumulators stay in the accumulation registers, the vector registers are for the stages
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                asm volatile("" : "+a"(lacc[nt]));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+a"(oacc[mt][nt]));
            }
        };
        pn_kbuf<HD> k0, k1;
        pn_vbuf<HD> v0, v1;
        __builtin_amdgcn_sched_barrier(0);
        ldk(k0, 0);
        __builtin_amdgcn_sched_barrier(0);
        ldv(v0, 0);
        __builtin_amdgcn_sched_barrier(0);
        ldk(k1, 1);
        __builtin_amdgcn_sched_barrier(0);
        int i = 0;
        for (; i + 1 < n_all; i += 2) {             // (no way out in the middle: it would spoil the load counts)
            ldv(v1, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            block(k0, v0, i);
            ldv(v0, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            block(k1, v1, i + 1);
        }
        if (i < n_all) block(k0, v0, i);
    }
    __syncthreads();             // every wave is done with the query tile: LDS changes hands

    // the waves' (max, sum, O) side by side in LDS, combined by all threads.  oacc[x*2*VW + u][nt][j]:
    // query row nt*16 + c, feature (x*16 + 4g + j) * VF + u
    float* s_o = reinterpret_cast<float*>(smem);                               // [waves][ROWS][OROW]
    float2* s_ml = reinterpret_cast<float2*>(s_o + PN_WAVES * ROWS * OROW);    // [waves][ROWS]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = wave * ROWS + nt * 16 + c;
        if (g == 0) s_ml[n] = make_float2(m_run[nt], lacc[nt][0]);
#pragma unroll
        for (int x = 0; x < VL; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int u = 0; u < VF; u += 4) {
                    const int mt = x * VF + u;
                    *reinterpret_cast<f32x4*>(&s_o[n * OROW + (x * 16 + 4 * g + j) * VF + u]) =
                        (f32x4){oacc[mt][nt][j], oacc[mt + 1][nt][j], oacc[mt + 2][nt][j], oacc[mt + 3][nt][j]};
                }
    }
    __syncthreads();
    pa_finish<PN_WAVES, HD, ROWS, bf16_t>(D, A, P, K, kvh, n_rows, s_o, s_ml, tid, 64 * PN_WAVES);
}

// As cs_load_to_lds, where the base comes straight from a lane: five wait states lie between a
// v_readlane and the load that takes its address from the result.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void cs_load_to_lds_lane(unsigned voff, const void* sbase, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(lds_addr) : "m0");
}
#pragma clang diagnostic pop

// ---- many query rows: the matrix cores and the vector unit are the bound -----------------------------
// Eight waves have 16 * NT query rows each and walk the tokens together: every 32-token block goes once
// from its pages to LDS and serves all of them.  Each wave requests its share of a block (1 KB pieces,
// direct to LDS) into a ring of stages, so several blocks are in flight while one is multiplied; the
// requests and the waits on them are counted exactly, by hand, and the kernel has no other vector
// memory load in its loop but the page numbers of the next 64 blocks.
//   keys: one piece = 16 tokens x 32 features in fragment order, a lane's 16 bytes are what it multiplies
//   values: one piece = 16 tokens x 32 features as two 16 x 16 squares of 32-byte rows, which the transposing LDS read
//   (four tokens of one feature per lane) takes apart without bank conflicts
// The products, the softmax and the order of tokens in the probabilities are those of the kernel above.
// What bounds it: the matrix units are busy 46 % of the time and the vector units 45 % (a block of 32
// tokens and 32 rows is 544 cycles of products and 500 of softmax), and little of either overlaps; at
// that rate the card is near its power limit (all zeros: 20 % faster).  Calls one after the other,
// median and range: 4096 rows of 32 heads on an empty cache 150 us (146 to 167) = 0.92 PFLOP/s; 2048
// rows behind 16384 tokens, with the merge, 538 us (531 to 612) = 1.09; 16 streams of 33 rows of 28
// heads (231 of 256 tile rows) behind 65535 tokens, with the merge, 608 us (600 to 645) = 0.82.  Under
// the profiler, which spaces the launches, the kernel alone takes about 180, 620 and 700 us at the
// median (0.76, 0.94 and 0.71).  Tried against this, same card: no teams +3 %, no wave
// priorities +1 to 2.5 %; the products of the next block woven into the softmax by hand +10 %;
// fragments of a whole block read ahead +3 to 5 %; 64 rows a wave in four waves: spills; two workgroups
// of four waves per compute unit: the same at 4096 rows, +20 % where one tile's rows had become two's.
#define PW_WAVES 8
template <int HD, int NT>
__global__ __launch_bounds__(64 * PW_WAVES) void k_paged_wide(cs_pages_dev D, pa_args A, pa_plan P) {
    constexpr int KS = HD / 32, MT = HD / 16;
    constexpr int WROWS = 16 * NT, TR = PW_WAVES * WROWS;
    constexpr int NLOAD = 4 * KS, LD = NLOAD / PW_WAVES;       // pieces of a block; per wave
    constexpr int STAGE_BYTES = NLOAD * 1024, V_AT = 2 * KS * 1024;
    constexpr int STAGES = HD == 256 ? 5 : 8;
    static_assert(NLOAD % PW_WAVES == 0 && STAGES * STAGE_BYTES <= 160 * 1024, "every wave the same number of requests; LDS");
    __shared__ __attribute__((aligned(16))) unsigned char stage[STAGES][STAGE_BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int KVH = D.p.n_kv_heads;
    // KV heads in turn, so that with eight of them each stays on one die and its cache
    const unsigned wg = cs_paged_wg();
    const int kvh = wg % KVH;
    pa_work K;
    if (!pa_find(D, A.G, A.window, P, wg / KVH, kvh, K)) return;
    const pa_tile& T = K.T;
    const int hd = D.p.head_dim, G = A.G;
    const int n_rows = min(TR, T.QR - T.n0);
    const int i_lo = T.n0 / G, i_hi = (T.n0 + n_rows - 1) / G;
    const int n_lim = min(T.L + i_hi + 1, D.cap);              // tokens that the tile's last row sees
    const int n_tok = min(T.L + T.rows, D.cap);                // tokens that are there
    const int w_first = A.window ? T.L + i_lo - A.window + 1 : 0;       // tokens before it are seen by no row of the tile
    const int base = A.window ? max(0, T.L + i_lo - A.window + 1) & ~31 : 0;
    const int w_begin = (int)min((int64_t)base + (int64_t)K.split * K.chunk, (int64_t)n_lim);
    const int t_end = K.split == K.nsplit - 1 ? n_lim : (int)min((int64_t)w_begin + K.chunk, (int64_t)n_lim);
    const int nblocks = (t_end - w_begin + 31) / 32;

    // query fragments, once; they must have arrived before the first counted request
    const int n0 = T.n0 + wave * WROWS + c;
    bf16x8 qreg[NT][KS];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = n0 + nt * 16, i = n / G;
        const bf16_t* qp = (const bf16_t*)A.q + (T.row0 + i) * A.q_row + (kvh * G + n - i * G) * A.q_head + g * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s)
            qreg[nt][s] = n < T.QR && s * 32 + g * 8 < hd ? *reinterpret_cast<const bf16x8*>(qp + s * 32) : (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qreg[nt][s]));

    // this wave's pieces: id = wave + 8u; below 2*KS keys (half id / KS, features 32 * (id % KS) ..),
    // above values likewise.  Features that the head does not have are read at feature 0: their query
    // elements are 0, their outputs are not stored.
    unsigned voff[LD];
#pragma unroll
    for (int u = 0; u < LD; ++u) {
        const int id = wave + PW_WAVES * u, v = id >= 2 * KS, x = id % KS;
        const int token = v ? (lane & 31) >> 1 : c;
        const int feature = x * 32 + (v ? (lane >> 5) * 16 + (lane & 1) * 8 : g * 8);
        voff[u] = token * (unsigned)(v ? D.p.v_token : D.p.k_token) * 2 + (feature < hd ? feature * 2 : 0);
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&stage[0][0];

    // A lane has one of the next 64 blocks: where in the pool each of the wave's pieces of it starts,
    // so that a request costs the scalar unit no multiplication.  A half whose page does not exist is
    // read from page 0 and masked: from a whole half of it, also where a range that lies behind all its
    // tile sees begins at a token that is no multiple of 16.
    const int32_t* tab = D.p.table + T.b * D.p.table_stride;
    unsigned from_lo[LD], from_hi[LD];
    unsigned long long okay0 = 0, okay1 = 0, old0 = 0, old1 = 0;     // halves that exist, of these and of the 64 blocks before
    auto pages = [&](int blk0) {
        const int64_t t = (int64_t)w_begin + 32 * ((int64_t)blk0 + lane);
        int page0 = -1, page1 = -1;
        if (t < t_end) {
            page0 = tab[t >> D.page_log2];
            const int e = (int)((t + 16) >> D.page_log2);
            page1 = e < D.p.table_pages ? tab[e] : -1;
        }
        const bool ok0 = (unsigned)page0 < (unsigned)D.p.n_pages, ok1 = (unsigned)page1 < (unsigned)D.p.n_pages;
        old0 = okay0, old1 = okay1;
        okay0 = __ballot(ok0), okay1 = __ballot(ok1);
#pragma unroll
        for (int u = 0; u < LD; ++u) {
            const int id = wave + PW_WAVES * u, v = id >= 2 * KS, half = id / KS & 1;
            const int page = half ? (ok1 ? page1 : 0) : (ok0 ? page0 : 0), slot = (int)(t + 16 * half) & (D.p.page_size - 16);
            const int64_t at = v ? page * D.p.v_page + kvh * D.p.v_head + slot * D.p.v_token : page * D.p.k_page + kvh * D.p.k_head + slot * D.p.k_token;
            const uint64_t from = (uint64_t)(v ? D.p.v : D.p.k) + 2 * at;
            from_lo[u] = (unsigned)from;
            from_hi[u] = (unsigned)(from >> 32);
        }
    };
    auto issue = [&](int blk, int st) {
#pragma unroll
        for (int u = 0; u < LD; ++u) {
            const uint64_t from = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)from_hi[u], blk & 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)from_lo[u], blk & 63);
            cs_load_to_lds_lane(voff[u], (const void*)from, lds0 + st * STAGE_BYTES + (wave + PW_WAVES * u) * 1024);
        }
    };
    // At most INFLIGHT of this wave's requests still in flight, then meet the other waves.  The two
    // waves of a SIMD meet them at different points of a block: the first four behind it, the others
    // between scores and softmax, so that one wave of every SIMD has the matrix unit while the other
    // has the vector unit.  (One statement: see cs_load_to_lds_if.)
    constexpr int INFLIGHT = LD * (STAGES - 3);
    const int team = wave / (PW_WAVES / 2);
#define PW_SYNC(on) \
    asm volatile("s_cmp_eq_u32 %1, 0\n\ts_cbranch_scc1 .Lno%=\n\ts_waitcnt vmcnt(%0)\n\ts_barrier\n.Lno%=:" ::"n"(INFLIGHT), "s"(on) : "memory", "scc")

    f32x4 oacc[MT][NT], lacc[NT];
    float m_run[NT], thr[NT];
    int q_last[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int i = (n0 + nt * 16) / G;
        q_last[nt] = T.L + i;
        m_run[nt] = thr[nt] = -INFINITY;
        lacc[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = A.scale2, inv_scale2 = 1.0f / A.scale2;
    const bf16_t one = (bf16_t)1.0f;
    const bf16x8 ones = (bf16x8){one, one, one, one, one, one, one, one};

    auto scores = [&](const unsigned char* sp, f32x4 (&sacc)[2][NT]) {
        auto k_frag = [&](int a, int s) { return *reinterpret_cast<const bf16x8*>(sp + ((a * KS + s) * 64 + lane) * 16); };
        bf16x8 k0 = k_frag(0, 0), k1 = k_frag(1, 0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            bf16x8 m0 = k0, m1 = k1;
            if (s + 1 < KS) {
                m0 = k_frag(0, s + 1);
                m1 = k_frag(1, s + 1);
            }
            const f32x4 zero4 = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                sacc[0][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qreg[nt][s], s == 0 ? zero4 : sacc[0][nt], 0, 0, 0);
                sacc[1][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qreg[nt][s], s == 0 ? zero4 : sacc[1][nt], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            k0 = m0;
            k1 = m1;
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // the running maximum of the tile rows moves (and O is rescaled) only when it is left behind by 2^8
    auto reference = [&](const f32x4 (&sacc)[2][NT], bool masked) {
        if (!masked) {
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float lm = fmaxf(fmaxf(fmaxf(sacc[0][nt][0], sacc[0][nt][1]), fmaxf(sacc[0][nt][2], sacc[0][nt][3])),
                                       fmaxf(fmaxf(sacc[1][nt][0], sacc[1][nt][1]), fmaxf(sacc[1][nt][2], sacc[1][nt][3])));
                over |= !(lm <= thr[nt]);
            }
            if (!__any(over)) return;
        }
        bool moved = false;
        float alpha[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = fmaxf(fmaxf(sacc[0][nt][0], sacc[0][nt][1]), sacc[0][nt][2]);
            mx = fmaxf(fmaxf(mx, sacc[0][nt][3]), sacc[1][nt][0]);
            mx = fmaxf(fmaxf(mx, sacc[1][nt][1]), fmaxf(sacc[1][nt][2], sacc[1][nt][3]));
            mx = fa_row4_max(mx) * scale2;
            const bool up = mx > m_run[nt] + FA_RESCALE_LOG2;
            const float m_new = up ? mx : m_run[nt];
            alpha[nt] = up ? __builtin_amdgcn_exp2f(m_run[nt] - (m_new == -INFINITY ? 0.f : m_new)) : 1.0f;
            moved |= up;
            m_run[nt] = m_new;
            thr[nt] = m_new == -INFINITY ? -INFINITY : (m_new + FA_RESCALE_LOG2) * inv_scale2;
        }
        if (__any(moved)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                lacc[nt] *= alpha[nt];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] *= alpha[nt];
            }
        }
    };
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    auto finish = [&](f32x4 (&sacc)[2][NT], const unsigned char* sp, int t0, auto masked_tag, bool ok0, bool ok1) {
        constexpr bool MASKED = decltype(masked_tag)::value;
        if (MASKED) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = t0 + 16 * a + 4 * g + j;
                        const bool sees = t <= q_last[nt] && (A.window == 0 || t > q_last[nt] - A.window) && t < n_tok && (a ? ok1 : ok0);
                        sacc[a][nt][j] = sees ? sacc[a][nt][j] : -INFINITY;
                    }
        }
        reference(sacc, MASKED);
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pb[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float m_safe = m_run[nt] == -INFINITY ? 0.f : m_run[nt];
#pragma unroll
            for (int e = 0; e < 8; ++e) pb[nt][e] = (bf16_t)__builtin_amdgcn_exp2f(fmaf(sacc[e >> 2][nt][e & 3], scale2, -m_safe));
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 vf[4];
        auto v_frag = [&](int mt) {
            s16x4 h[2];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const unsigned char* p = sp + V_AT + (a * KS + (mt >> 1)) * 1024 + (mt & 1) * 512 + lane * 8;
                h[a] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) unsigned char*)p);
                if (MASKED) {
                    // what lies behind the last token, in place of a page or before every window may be
                    // anything, and 0 * anything must stay 0
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = t0 + 16 * a + 4 * g + j;
                        if (t >= n_tok || t < w_first || !(a ? ok1 : ok0)) h[a][j] = 0;
                    }
                }
            }
            return __builtin_bit_cast(bf16x8, (s16x8){h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]});
        };
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int mt = 0; mt < 3; ++mt) vf[mt] = v_frag(mt);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt + 3 < MT) vf[(mt + 3) & 3] = v_frag(mt + 3);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) oacc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mt & 3], pb[nt], oacc[mt][nt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) lacc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[nt], lacc[nt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
    };

    // Blocks 0 .. STAGES-3 are requested up front; round i requests block i + STAGES - 2 into the stage
    // of block i - 2, whose values the second team has read before the meeting behind its scores of
    // block i - 1.  Behind round i's meeting block i + 1 is there.
    pages(0);
#pragma unroll
    for (int j = 0; j < STAGES - 2; ++j) issue(j, j);         // (past the last block: page 0, into a stage that nobody reads)
    PW_SYNC(1);
    int st_cur = 0, st_req = STAGES - 2;
    // The loop's bound and the position come from a vector register that the compiler cannot see
    // through: around branches it takes for uniform it splits the live ranges of the accumulators,
    // copies and spills them.
    int vzero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(vzero));
    const int nblocks_v = nblocks + vzero;
    // positions that this wave's rows have: blocks outside what they see are not computed, blocks
    // inside need no mask
    const int p_lo = T.L + (T.n0 + wave * WROWS) / G + vzero;
    const int p_hi = T.L + min(T.rows - 1, (T.n0 + wave * WROWS + WROWS - 1) / G) + vzero;
    // tokens below w_lo are seen by no row of the wave, those from w_hi on by every one (as far as a
    // window goes)
    const int w_lo = A.window ? p_lo - A.window + 1 : 0, w_hi = A.window ? p_hi - A.window + 1 : 0;
    const int p_end = T.n0 + wave * WROWS < T.QR ? p_hi : -1;      // a wave without rows multiplies nothing
    const int p_open = min(p_lo, D.cap - 1);
    const std::integral_constant<bool, false> plain_tag;
    const std::integral_constant<bool, true> masked_tag;
    f32x4 sa[2][NT];
    for (int i = 0; i < nblocks_v; ++i) {
        const int ahead = i + STAGES - 2;
        if ((ahead & 63) == 0) pages(ahead);
        issue(ahead, st_req);
        st_req = st_req + 1 == STAGES ? 0 : st_req + 1;
        const int t0 = w_begin + i * 32;
        const unsigned long long whole = (ahead >> 6) == (i >> 6) ? okay0 & okay1 : old0 & old1;
        const int gone = 1 - ((int)(whole >> (i & 63)) & 1) + vzero;
        const bool mine = (t0 <= p_end) & (t0 + 31 >= w_lo);
        if (mine) scores(stage[st_cur], sa);
        PW_SYNC(team);
        if (mine) {
            if ((t0 + 31 > p_open) | (t0 < w_hi) | (gone != 0)) {
                const unsigned long long h0 = (ahead >> 6) == (i >> 6) ? okay0 : old0, h1 = (ahead >> 6) == (i >> 6) ? okay1 : old1;
                finish(sa, stage[st_cur], t0, masked_tag, (int)(h0 >> (i & 63)) & 1, (int)(h1 >> (i & 63)) & 1);
            } else finish(sa, stage[st_cur], t0, plain_tag, true, true);
        }
        st_cur = st_cur + 1 == STAGES ? 0 : st_cur + 1;
        PW_SYNC(1 - team);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // surplus requests, before the LDS is given up
#undef PW_SYNC

    // oacc[mt][nt][j]: query row nt*16 + c, feature mt*16 + 4g + j
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = n0 + nt * 16;
        if (n >= T.QR) continue;
        const int i = n / G, h = kvh * G + n - i * G;
        const int64_t r = T.row0 + i;
        const float l = lacc[nt][0];
        if (K.nsplit == 1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int d = mt * 16 + 4 * g;
                if (d < hd) pa_store4((bf16_t*)A.out + r * A.out_row + h * A.out_head + d, oacc[mt][nt] * inv);
            }
            continue;
        }
        const int64_t at = ((int64_t)K.entry * KVH + kvh) * P.TR + n - T.n0;
        if (g == 0) P.pml[at] = make_float2(m_run[nt], l);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int d = mt * 16 + 4 * g;
            if (d < hd) *reinterpret_cast<f32x4*>(P.po + at * hd + d) = oacc[mt][nt];
        }
    }
}

// ---- float32 caches: everything in float32, on the float32 matrix instruction -------------------------
//   S^T[token][row] = K . Q^T, O^T[feature][row] += V^T . P^T over blocks of 16 tokens, four k per instruction.
// Lane (c, g) loads 16 bytes of a key row, four steps of the first product; the rows of S^T that it
// gets are the k of the second one, step j taking token 4g + j, and its 16 bytes of that token's value
// row are four features 4c + u, one for each of four tiles.  So nothing is moved between lanes, and
// nothing goes through LDS but the query rows (and, with TOKENS, the waves' results: few rows, where
// the waves share them and take the token blocks in turn; without it every wave has 16 * NT rows of its
// own, and what bounds it is the instruction's rate, 157 TFLOP/s, the re-read blocks coming out of the
// caches).  Two workgroups share a compute unit, and the matrix units are busy 74 % while they do: two
// streams of 700 and 438 rows behind 3001 and 1876 tokens, 8 heads of 128: 150 to 155 us = 86 to 89
// TFLOP/s (one workgroup per compute unit: 225 us; 16 rows a wave: 4 to 9 % slower; two key blocks
// ahead: no change).  Few rows are bound by memory: 8 single tokens behind 8000, 8 heads of 128, 524
// MB: 90 to 94 us = 5.6 to 5.8 TB/s, 95 us with the merge.
#define PF_WAVES 4
template <int HD, int NT, bool TOKENS>
__global__ __launch_bounds__(64 * PF_WAVES, !TOKENS && HD <= 128 ? 2 : 1) void k_paged_f32(cs_pages_dev D, pa_args A, pa_plan P) {
    constexpr int KL = HD / 16, VX = HD / 64, MT = HD / 16;
    constexpr int WROWS = 16 * NT, TR = TOKENS ? WROWS : PF_WAVES * WROWS, OROW = HD + 4, QROW = HD + 4;
    constexpr int MERGE_FLOATS = TOKENS ? PF_WAVES * WROWS * (OROW + 2) : 0, Q_FLOATS = TR * QROW;
    __shared__ __attribute__((aligned(16))) float smem[MERGE_FLOATS > Q_FLOATS ? MERGE_FLOATS : Q_FLOATS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const unsigned wg = cs_paged_wg();
    const int KVH = D.p.n_kv_heads, kvh = wg % KVH;
    pa_work K;
    if (!pa_find(D, A.G, A.window, P, wg / KVH, kvh, K)) return;
    const pa_tile& T = K.T;
    const int hd = D.p.head_dim, G = A.G;
    const int n_rows = min(TR, T.QR - T.n0);
    const int i_hi = (T.n0 + n_rows - 1) / G;
    const int n_lim = min(T.L + i_hi + 1, D.cap);
    const int base = A.window ? max(0, T.L + T.n0 / G - A.window + 1) & ~31 : 0;
    const int w_begin = (int)min((int64_t)base + (int64_t)K.split * K.chunk, (int64_t)n_lim);
    const int t_end = K.split == K.nsplit - 1 ? n_lim : (int)min((int64_t)w_begin + K.chunk, (int64_t)n_lim);
    for (int idx = tid; idx < TR * (HD / 4); idx += 64 * PF_WAVES) {
        const int n = idx / (HD / 4), d = idx % (HD / 4) * 4;
        f32x4 v = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (n < n_rows && d < hd) {
            const int i = (T.n0 + n) / G, h = kvh * G + T.n0 + n - i * G;
            v = *reinterpret_cast<const f32x4*>((const float*)A.q + (T.row0 + i) * A.q_row + h * A.q_head + d);
        }
        *reinterpret_cast<f32x4*>(&smem[n * QROW + d]) = v;
    }
    const int wrow = TOKENS ? 0 : wave * WROWS;         // the wave's first row in the tile
    const int w_rows = max(0, min(WROWS, n_rows - wrow));
    // positions of the wave's first and last row, tokens that it walks
    const int p_lo = T.L + (T.n0 + wrow) / G, p_hi = T.L + (T.n0 + wrow + max(w_rows, 1) - 1) / G;
    const int my_end = w_rows ? min(t_end, min(p_hi + 1, D.cap)) : w_begin;
    const int open_lo = A.window ? p_hi - A.window + 1 : 0, open_hi = min(p_lo + 1, D.cap);
    const int w_first = A.window ? T.L + T.n0 / G - A.window + 1 : 0;   // tokens before it are seen by no row of the tile
    int q_last[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = wrow + nt * 16 + c;
        q_last[nt] = n < n_rows ? T.L + (T.n0 + n) / G : -1;
    }
    const float* Kh = (const float*)D.p.k + kvh * D.p.k_head;
    const float* Vh = (const float*)D.p.v + kvh * D.p.v_head;
    const int32_t* tab = D.p.table + T.b * D.p.table_stride;
    constexpr unsigned NOWHERE = 0x80000000u;
    const unsigned kts = (unsigned)D.p.k_token * 4, vts = (unsigned)D.p.v_token * 4;
    unsigned koff[KL], voff[4][VX];
#pragma unroll
    for (int s = 0; s < KL; ++s) koff[s] = s * 16 + g * 4 < hd ? c * kts + s * 64 + g * 16 : NOWHERE;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < VX; ++x) voff[j][x] = x * 64 + c * 4 < hd ? (4 * g + j) * vts + x * 256 + c * 16 : NOWHERE;

    f32x4 oacc[MT][NT];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = -INFINITY;
        l_run[nt] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = A.scale2;
    __syncthreads();

    constexpr int STEP = TOKENS ? 16 * PF_WAVES : 16;
    for (int seg0 = w_begin; seg0 < t_end; seg0 += 64 * STEP) {
        const int t_begin = seg0 + (TOKENS ? 16 * wave : 0);
        const int n_all = t_begin < my_end ? min(64, (my_end - t_begin + STEP - 1) / STEP) : 0;
        int page_l = -1;
        {
            const int64_t tb = (int64_t)t_begin + (int64_t)lane * STEP;
            if (tb < my_end) page_l = tab[tb >> D.page_log2];
            page_l = (unsigned)page_l < (unsigned)D.p.n_pages ? page_l : -1;
        }
        auto at = [&](int i) { return t_begin + i * STEP; };
        auto page_of = [&](int i) { return __builtin_amdgcn_readlane(page_l, i); };
        auto buffer = [&](const float* head, int64_t page_stride, unsigned ts, int i) {
            const int t = at(i), page = i < n_all ? page_of(i) : -1, live = min(16, n_lim - t);
            const unsigned bytes = page >= 0 && live > 0 ? (live - 1) * ts + hd * 4 : 0;
            const char* p = (const char*)(head + (page >= 0 ? page : 0) * page_stride) + (int64_t)(t & (D.p.page_size - 1)) * ts;
            return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, CS_BUFFER_WORD3);
        };
        auto ldk = [&](f32x4 (&buf)[KL], int i) {
            const auto rs = buffer(Kh, D.p.k_page, kts, i);
#pragma unroll
            for (int s = 0; s < KL; ++s) buf[s] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, koff[s], 0, 0));
        };
        auto ldv = [&](f32x4 (&buf)[4][VX], int i) {
            const auto rs = buffer(Vh, D.p.v_page, vts, i);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < VX; ++x) buf[j][x] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, voff[j][x], 0, 0));
        };
        auto block = [&](f32x4 (&kb)[KL], f32x4 (&vb)[4][VX], int i) {
            f32x4 sacc[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sacc[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            f32x4 odd[NT];                              // a second chain, where one would wait for itself
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) odd[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KL; ++s) {
                f32x4 qb[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) qb[nt] = *reinterpret_cast<const f32x4*>(&smem[(wrow + nt * 16 + c) * QROW + s * 16 + g * 4]);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        f32x4& z = u & 1 ? odd[nt] : sacc[nt];
                        z = __builtin_amdgcn_mfma_f32_16x16x4f32(kb[s][u], qb[nt][u], z, 0, 0, 0);
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sacc[nt] += odd[nt];
            __builtin_amdgcn_sched_barrier(0);
            ldk(kb, i + (TOKENS ? 2 : 1));
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = at(i), page = page_of(i);
            if (t0 < open_lo || t0 + 16 > open_hi || page < 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = t0 + 4 * g + j;
                        const bool sees = t <= q_last[nt] && (A.window == 0 || t > q_last[nt] - A.window) && t < D.cap && page >= 0;
                        sacc[nt][j] = sees ? sacc[nt][j] : -INFINITY;
                    }
                if (t0 < w_first) {                     // (what has left every window may be anything, and 0 * anything must stay 0)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int x = 0; x < VX; ++x)
#pragma unroll
                            for (int u = 0; u < 4; ++u) vb[j][x][u] = t0 + 4 * g + j < w_first ? 0.f : vb[j][x][u];
                }
            }
            bool moved = false;
            float alpha[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float mx = fa_row4_max(fmaxf(fmaxf(sacc[nt][0], sacc[nt][1]), fmaxf(sacc[nt][2], sacc[nt][3]))) * scale2;
                const bool up = mx > m_run[nt] + FA_RESCALE_LOG2;
                const float m_new = up ? mx : m_run[nt];
                const float m_safe = m_new == -INFINITY ? 0.f : m_new;
                alpha[nt] = up ? __builtin_amdgcn_exp2f(m_run[nt] - m_safe) : 1.0f;
                moved |= up;
                m_run[nt] = m_new;
#pragma unroll
                for (int j = 0; j < 4; ++j) sacc[nt][j] = __builtin_amdgcn_exp2f(fmaf(sacc[nt][j], scale2, -m_safe));
            }
            if (__any(moved)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    l_run[nt] *= alpha[nt];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] *= alpha[nt];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) l_run[nt] += (sacc[nt][0] + sacc[nt][1]) + (sacc[nt][2] + sacc[nt][3]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int x = 0; x < VX; ++x)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            oacc[x * 4 + u][nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vb[j][x][u], sacc[nt][j], oacc[x * 4 + u][nt], 0, 0, 0);
            if constexpr (!TOKENS) {
                __builtin_amdgcn_sched_barrier(0);
                ldv(vb, i + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        f32x4 k0[KL], v0[4][VX];
        __builtin_amdgcn_sched_barrier(0);
        ldk(k0, 0);
        __builtin_amdgcn_sched_barrier(0);
        ldv(v0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!TOKENS) {                        // either product covers the loads for the other: one buffer each
            for (int i = 0; i < n_all; ++i) block(k0, v0, i);
            continue;
        }
        f32x4 k1[KL], v1[4][VX];
        ldk(k1, 1);
        __builtin_amdgcn_sched_barrier(0);
        int i = 0;
        for (; i + 1 < n_all; i += 2) {
            ldv(v1, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            block(k0, v0, i);
            ldv(v0, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            block(k1, v1, i + 1);
        }
        if (i < n_all) block(k0, v0, i);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {                   // a row's sum is spread over its four lanes
        l_run[nt] += __shfl_xor(l_run[nt], 16, 64);
        l_run[nt] += __shfl_xor(l_run[nt], 32, 64);
    }
    // oacc[x*4 + u][nt][j]: query row nt*16 + c, feature x*64 + 16g + 4j + u
    if constexpr (TOKENS) {
        __syncthreads();
        float* s_o = smem;
        float2* s_ml = reinterpret_cast<float2*>(s_o + PF_WAVES * WROWS * OROW);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = wave * WROWS + nt * 16 + c;
            if (g == 0) s_ml[n] = make_float2(m_run[nt], l_run[nt]);
#pragma unroll
            for (int x = 0; x < VX; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<f32x4*>(&s_o[n * OROW + x * 64 + 16 * g + 4 * j]) =
                        (f32x4){oacc[x * 4][nt][j], oacc[x * 4 + 1][nt][j], oacc[x * 4 + 2][nt][j], oacc[x * 4 + 3][nt][j]};
        }
        __syncthreads();
        pa_finish<PF_WAVES, HD, WROWS, float>(D, A, P, K, kvh, n_rows, s_o, s_ml, tid, 64 * PF_WAVES);
    } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = wrow + nt * 16 + c;
            if (n >= n_rows) continue;
            const int i = (T.n0 + n) / G, h = kvh * G + T.n0 + n - i * G;
            const int64_t r = T.row0 + i, at = ((int64_t)K.entry * KVH + kvh) * P.TR + n;
            const bool whole = K.nsplit == 1;
            const float inv = l_run[nt] > 0.f ? 1.0f / l_run[nt] : 0.f;
            if (g == 0 && !whole) P.pml[at] = make_float2(m_run[nt], l_run[nt]);
#pragma unroll
            for (int x = 0; x < VX; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int d = x * 64 + 16 * g + 4 * j;
                    const f32x4 o = (f32x4){oacc[x * 4][nt][j], oacc[x * 4 + 1][nt][j], oacc[x * 4 + 2][nt][j], oacc[x * 4 + 3][nt][j]};
                    if (d >= hd) continue;
                    if (whole) pa_store4((float*)A.out + r * A.out_row + h * A.out_head + d, o * inv);
                    else pa_store4(P.po + at * hd + d, o);
                }
        }
    }
}

// ---- joining token ranges ---------------------------------------------------------------------
// out[r][h] = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.  2^lanes_log2 lanes have a query row's hd
// features, four each; a lane reads the (max, sum) pairs of every lanes-th range, and the weights go
// round by shuffles.  The workgroups are those of the kernel before it: the ones that had the ranges of
// a tile share out its rows (4 ranges of 8 x 44 rows and 8 heads: 6 us, a launch's own 3 among them; 13
// ranges of 37 float32 tiles and 2 heads, 962 workgroups, 11.6 us).
#define PM_THREADS 256
template <typename T_>
__global__ __launch_bounds__(PM_THREADS) void k_paged_merge(cs_pages_dev D, pa_args A, pa_plan P, int lanes_log2) {
    const int KVH = D.p.n_kv_heads, kvh = blockIdx.x % KVH;
    const int entry = blockIdx.x / KVH;
    const int4 who = P.who[entry];
    const int split = who.w & 0xffff, nsplit = who.w >> 16;
    if (nsplit <= 1) return;
    const int lanes = 1 << lanes_log2, sub = threadIdx.x & (lanes - 1), d = sub * 4, per = PM_THREADS >> lanes_log2, hd = D.p.head_dim;
    const int64_t step = (int64_t)KVH * P.TR;                      // from one range's row to the next one's
    for (int n = split * per + (threadIdx.x >> lanes_log2); n < P.TR && who.y + n < who.z; n += nsplit * per) {
        const int64_t at = ((int64_t)(entry - split) * KVH + kvh) * P.TR + n;
        float M = -INFINITY;
        for (int s = sub; s < nsplit; s += lanes) M = fmaxf(M, P.pml[at + s * step].x);
        for (int o = lanes >> 1; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
        const float Ms = M == -INFINITY ? 0.f : M;
        f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        for (int s0 = 0; s0 < nsplit; s0 += lanes) {
            float2 ml = make_float2(-INFINITY, 0.f);
            if (s0 + sub < nsplit) ml = P.pml[at + (s0 + sub) * step];
            const float w = __builtin_amdgcn_exp2f(ml.x - Ms), wl = w * ml.y;
            const int ns = min(lanes, nsplit - s0);
            const float* __restrict__ src = P.po + (at + s0 * step) * hd + min(d, hd - 4);
            for (int s = 0; s < ns; s += 4)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    // (past the last range: weight 0, its row once more; a range that saw nothing has
                    // stored zeros)
                    const int from = (threadIdx.x & 63 & ~(lanes - 1)) + min(s + u, ns - 1);
                    const float keep = s + u < ns ? 1.f : 0.f;
                    l += keep * __shfl(wl, from, 64);
                    acc += keep * __shfl(w, from, 64) * *reinterpret_cast<const f32x4*>(src + min(s + u, ns - 1) * step * hd);
                }
        }
        const int i = (who.y + n) / A.G, h = kvh * A.G + who.y + n - i * A.G;
        if (d < hd) pa_store4((T_*)A.out + (int64_t)(who.x + i) * A.out_row + h * A.out_head + d, acc * (l > 0.f ? 1.0f / l : 0.f));
    }
}

// ---- entry points --------------------------------------------------------------------------
static int check_shape(const char* who, const cs_pages* p, int32_t n_heads, int32_t R, int32_t max_rows, int64_t max_len) {
    CS_TRY(cs_check_pages(who, p));
    CS_REQUIRE(n_heads >= 1 && n_heads <= 4096 && n_heads % p->n_kv_heads == 0, CS_E_ARG,
               "%s: n_heads must be a multiple of n_kv_heads, up to 4096", who);
    CS_REQUIRE(R >= 0 && R <= 1 << 26, CS_E_ARG, "%s: R out of range", who);
    CS_REQUIRE((int64_t)R * n_heads <= 1 << 30, CS_E_UNSUPPORTED, "%s: R * n_heads exceeds 2^30", who);
    CS_REQUIRE(max_rows >= 0 && max_len >= 0, CS_E_ARG, "%s: negative max_rows or max_len", who);
    return CS_OK;
}

// How a call is cut: the same for the workspace and the launches.
struct pa_part {
    int nt, TR, qr_lo, qr_hi, tiles;          // tiles: an upper bound; 0: no launch
    int slots, start, join, n_max, step, chunk, entries;
};
struct pa_cut {
    int hdt;
    pa_part narrow, wide;
    int64_t at_w, bytes;                      // where the second launch's partial results start; bytes in all
};
#define PN_MOST 48                // query rows up to which a stream takes the kernel of few rows
#define PA_MOST_RANGES 256
// Pairs that there is room for beyond one per tile, in rounds of the chip.  With room for as many as
// even out the rounds best the partial results, which are the workspace, come to 2.1 GB (3968 rows of
// 32 heads over a table of 2^20 tokens); with eight rounds they stay under 0.5 GB.  The cut is the same
// where that was never used (2048 rows of 32 heads behind 129000 tokens, a table of 2^17: 1.1 GB ->
// 0.3, 3.8 ms); else the rounds are less even, and there is less to join: 11 x 252 float32 rows of 28
// heads behind 31225 tokens 9.75 -> 10.2 ms, a float32 block of 1251 rows of 64 heads beside 23 single
// tokens, all behind 273 to 1090: 1000 -> 784 us.
#define PA_MOST_ROUNDS 8
// The host's cut prices the ranges as the device does, with every stream as long as the longest;
// batches of more than 64 streams take it. For the others it says how many (tile, range) pairs there is
// room for: one round of the chip, or what the host's cut has. (A workgroup without a pair ends at
// once, but where one fills a compute unit it waits for its turn.)
static int64_t pa_ranges(pa_part& t, int64_t len, int B, int KVH, int hd, int slots, int start, int join) {
    if (!t.tiles) return 0;
    t.slots = slots, t.start = start, t.join = join;
    const int64_t items = (int64_t)t.tiles * KVH;
    // (no ranges where the chip is full twice over, or where none would pay for the merge if they all
    // ran at once)
    const int ranges = (int)std::max<int64_t>(1, std::min<int64_t>(PA_MOST_RANGES, len / 64));
    bool one = items >= 2 * slots;
    if (items <= slots) {
        bool pays = false;
        for (int n = 2; n <= ranges && !pays; ++n) pays = cs_round_up(cs_ceil_div(len, n), 32) + join + n < cs_round_up(len, 32);
        one |= !pays;
    }
    const int most = one ? 1 : ranges;
    const int64_t room = t.tiles + cs_ceil_div((int64_t)PA_MOST_ROUNDS * slots, KVH);
    int64_t best = 0;
    int n_best = 1;
    for (int n = 1; n <= most && (n == 1 || B <= 64 || (int64_t)t.tiles * n <= room); ++n) {
        const int64_t chunk = cs_round_up(std::max<int64_t>(cs_ceil_div(len, n), 1), 32);
        const int64_t cost = cs_ceil_div(items * n, slots) * (chunk + start) + (n > 1 ? join + n : 0);
        if (n == 1 || cost < best) best = cost, n_best = n, t.chunk = (int)chunk;
    }
    t.entries = (int)std::min(room, std::max<int64_t>((int64_t)t.tiles * n_best, most > 1 && B <= 64 ? cs_ceil_div(slots, KVH) : 0));
    t.n_max = B > 64 ? n_best : std::min(most, t.entries);
    t.step = (int)cs_ceil_div(t.n_max, 64);
    return t.n_max > 1 ? cs_round_up((int64_t)t.entries * KVH * t.TR * (hd * 4 + 8), 16) + (int64_t)t.entries * 16 : 0;
}
static pa_cut pa_make_cut(const cs_pages* p, int H, bool has_row0, int R, int max_rows, int64_t max_len) {
    pa_cut c = {};
    const int KVH = p->n_kv_heads, G = H / KVH, B = p->batch, cap = p->table_pages * p->page_size;
    const int rows = has_row0 ? (max_rows ? std::min(max_rows, R) : R) : R / B;
    const int64_t qr = (int64_t)rows * G, all = (int64_t)R * G, len = max_len && max_len < cap ? max_len : cap;
    const bool f32 = p->dtype == CS_F32;
    c.hdt = p->head_dim <= 64 ? 64 : p->head_dim <= 128 ? 128 : 256;
    pa_part &N = c.narrow, &W = c.wide;
    // Streams of up to n_most query rows per KV head go to the kernel of few rows.  Where a batch has
    // longer ones too, that kernel is made for single tokens: a tile of 48 rows would cost every one of
    // them three tiles' products.
    const int n_most = c.hdt == 256 || qr > PN_MOST ? 16 : PN_MOST;
    if (has_row0 || qr <= n_most) {
        N.nt = (int)std::min<int64_t>(n_most / 16, cs_ceil_div(qr, 16));
        N.TR = 16 * N.nt;
        N.qr_hi = qr <= n_most ? 0x7fffffff : n_most;
        N.tiles = !has_row0 ? B : (int)(qr <= n_most ? all / N.TR + std::min(B, R) : std::min(B, R));
    }
    if (qr > n_most) {
        // Tiles of half the rows where whole ones, cut into ranges of 256 tokens of what a row sees on
        // average, leave the chip unfilled: a block of tokens takes such a tile about half as long, and
        // there are twice as many (6 streams of 985 rows of 4 heads: 60 -> 34 us; 1000 rows of 32
        // heads: 56 -> 35; 64 rows behind 4000 tokens: 28 -> 23; but 2 streams of 300 rows behind 1000:
        // 48 -> 52, by the rule whole).
        const bool unfilled = (all / (PW_WAVES * 32) + 1) * KVH * std::max<int64_t>(1, (len - rows / 2) / 256) < 256;
        W.nt = c.hdt == 256 || (!f32 && unfilled) ? 1 : 2;
        W.TR = (f32 ? PF_WAVES : PW_WAVES) * 16 * W.nt;
        W.qr_lo = has_row0 ? n_most : 0;
        W.qr_hi = 0x7fffffff;
        W.tiles = (int)(has_row0 ? all / W.TR + std::min<int64_t>(B, all / (n_most + 1)) : B * cs_ceil_div(qr, W.TR));
    }
    // The chip's slots: one workgroup per compute unit, two of the float32 kernel for many rows.  What
    // a workgroup's ends and the merge cost is in tokens of each kernel's own pace.  That of float32
    // blocks of few rows goes with the features, and so does what a merge costs in its tokens: 384 of
    // 64 features, 192 of 128, 96 of 256 (captured calls, one price of 512 for all before: a row each
    // of 4 streams behind 450, 8 heads of 128: 16.7 -> 12.5 us, behind 1000: 13.0 both; a row behind
    // 565, 8 heads of 256: 30.5 -> 17.1; 11 rows behind 565, 4 heads of 64: 11.9 -> 9.5, behind 450,
    // where it still does not pay, 11.4 both; called one by one from Python the last of these is bound
    // by its two launches instead of one, 11.8 -> 12.5).  The other three are single figures yet.
    // Against half and twice both of a kernel's, captured calls: few bfloat16 rows behind 600 to 900
    // tokens would gain 14 to 38 % from half where a token has 128 or 256 features and lose 6 to 16 %
    // where it has 64, behind 1000 to 1300 twice costs up to 131 %, and behind 2000 and more neither
    // changes 3 %; many bfloat16 rows on an empty cache take up to 2.6 times as long with half (2 x 600
    // rows of 28 heads: 26.6 -> 68 us), and twice changes them by -21 (2 x 600 behind 1000) to +10 %
    // (1500 rows of 8 heads of 64 behind 300); many float32 rows: -7 to +2 % with half, 3 % with twice.
    c.at_w = f32 ? pa_ranges(N, len, B, KVH, p->head_dim, 256, 128, 384 * 64 / c.hdt) : pa_ranges(N, len, B, KVH, p->head_dim, 256, 256, 768);
    c.bytes = c.at_w + (f32 ? pa_ranges(W, len, B, KVH, p->head_dim, 512, 16, 128) : pa_ranges(W, len, B, KVH, p->head_dim, 256, 128, 192));
    return c;
}

extern "C" int64_t cs_paged_attention_workspace(const cs_pages* p, int32_t n_heads, int32_t has_row0, int32_t R, int32_t max_rows,
                                                int64_t max_len) {
    const char* who = "cs_paged_attention_workspace";
    CS_TRY(check_shape(who, p, n_heads, R, max_rows, max_len));
    CS_REQUIRE(has_row0 || p->batch == 0 || R % p->batch == 0, CS_E_ARG, "%s: R rows cannot be shared out among %d streams without d_row0",
               who, p->batch);
    if (R == 0 || p->batch == 0) return 0;
    return pa_make_cut(p, n_heads, has_row0 != 0, R, max_rows, max_len).bytes;
}

template <int HD, int NT>
static int pn_launch(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s) {
    k_paged_narrow<HD, NT><<<grid, 64 * PN_WAVES, 0, s>>>(D, A, P);
    return cs_launch_ok("k_paged_narrow");
}
template <int HD, int NT, bool TOKENS>
static int pf_launch(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s) {
    k_paged_f32<HD, NT, TOKENS><<<grid, 64 * PF_WAVES, 0, s>>>(D, A, P);
    return cs_launch_ok("k_paged_f32");
}
template <int HD, int NT>
static int pw_launch(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s) {
    k_paged_wide<HD, NT><<<grid, 64 * PW_WAVES, 0, s>>>(D, A, P);
    return cs_launch_ok("k_paged_wide");
}
static pa_plan pa_plan_of(const pa_part& t, char* ws, int KVH, int hd) {
    const int64_t rows = (int64_t)t.entries * KVH * t.TR;
    float* po = (float*)ws;
    float2* pml = (float2*)(po + rows * hd);
    return {t.TR, t.qr_lo, t.qr_hi, t.slots, t.start, t.join, t.n_max, t.step, t.chunk, t.entries, po, pml,
            (int4*)(ws + cs_round_up(rows * (hd * 4 + 8), 16))};
}
static int pm_launch(const cs_pages_dev& D, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s) {
    if (P.n_max <= 1) return CS_OK;        // (with ranges a grid is some rounds of the chip: it needs x only)
    int lanes = 0;
    while (4 << lanes < D.p.head_dim) ++lanes;
    if (D.p.dtype == CS_F32) k_paged_merge<float><<<grid, PM_THREADS, 0, s>>>(D, A, P, lanes);
    else k_paged_merge<bf16_t><<<grid, PM_THREADS, 0, s>>>(D, A, P, lanes);
    return cs_launch_ok("k_paged_merge");
}

extern "C" int cs_paged_attention(const cs_pages* p, const void* q, int64_t q_row, int64_t q_head, int32_t n_heads,
                                  const int32_t* d_row0, int32_t R, float scale, int32_t window, int32_t max_rows,
                                  int64_t max_len, void* out, int64_t out_row, int64_t out_head, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
    const char* who = "cs_paged_attention";
    CS_TRY(check_shape(who, p, n_heads, R, max_rows, max_len));
    CS_REQUIRE(scale > 0.f && std::isfinite(scale), CS_E_ARG, "%s: scale must be positive and finite", who);
    CS_REQUIRE(window >= 0, CS_E_ARG, "%s: negative window", who);
    cs_pages_dev D;
    CS_TRY(cs_pages_view(who, p, d_row0, R, &D));
    if (R == 0 || p->batch == 0) return CS_OK;
    const size_t esz = p->dtype == CS_BF16 ? 2 : 4;
    CS_TRY(cs_check_rows(who, "q", q, q_row, q_head, esz));
    CS_TRY(cs_check_rows(who, "out", out, out_row, out_head, esz));
    CS_TRY(cs_check_apart(who, "out", out_row, R, out_head, n_heads, p->head_dim));
    pa_args A = {q, q_row, q_head, out, out_row, out_head, n_heads, n_heads / p->n_kv_heads, window, scale * 1.4426950408889634f};
    hipStream_t s = (hipStream_t)stream;
    const pa_cut c = pa_make_cut(p, n_heads, d_row0 != nullptr, R, max_rows, max_len);
    CS_REQUIRE(c.bytes <= 0 || (workspace && workspace_bytes >= c.bytes), CS_E_CAPACITY, "%s: the workspace has %lld bytes, %lld are needed",
               who, (long long)(workspace ? workspace_bytes : 0), (long long)c.bytes);
    CS_REQUIRE(((uintptr_t)workspace & 15) == 0, CS_E_ARG, "%s: the workspace is not aligned to 16 bytes", who);
    const int64_t grid_n = (int64_t)c.narrow.entries * p->n_kv_heads, grid_w = (int64_t)c.wide.entries * p->n_kv_heads;
    CS_REQUIRE(grid_n <= 0x7fffffff && grid_w <= 0x7fffffff, CS_E_UNSUPPORTED, "%s: too many tiles", who);
    const bool f32 = p->dtype == CS_F32;
    int rc = CS_OK;
    if (grid_w) {
        const pa_plan P = pa_plan_of(c.wide, (char*)workspace + c.at_w, p->n_kv_heads, p->head_dim);
        const dim3 n = cs_paged_grid(grid_w);
        if (f32) rc = c.hdt == 64 ? pf_launch<64, 2, false>(D, A, P, n, s) : c.hdt == 128 ? pf_launch<128, 2, false>(D, A, P, n, s) : pf_launch<256, 1, false>(D, A, P, n, s);
        else if (c.wide.nt == 2) rc = c.hdt == 64 ? pw_launch<64, 2>(D, A, P, n, s) : pw_launch<128, 2>(D, A, P, n, s);
        else rc = c.hdt == 64 ? pw_launch<64, 1>(D, A, P, n, s) : c.hdt == 128 ? pw_launch<128, 1>(D, A, P, n, s) : pw_launch<256, 1>(D, A, P, n, s);
        CS_TRY(rc);
        CS_TRY(pm_launch(D, A, P, n, s));
    }
    if (grid_n) {
        const pa_plan P = pa_plan_of(c.narrow, (char*)workspace, p->n_kv_heads, p->head_dim);
        const dim3 n = cs_paged_grid(grid_n);
#define PN(HD_, NT_) if (c.hdt == HD_ && c.narrow.nt == NT_) rc = f32 ? pf_launch<HD_, NT_, true>(D, A, P, n, s) : pn_launch<HD_, NT_>(D, A, P, n, s)
        PN(64, 1); PN(64, 2); PN(64, 3); PN(128, 1); PN(128, 2); PN(128, 3); PN(256, 1);
#undef PN
        CS_TRY(rc);
        CS_TRY(pm_launch(D, A, P, n, s));
    }
    return CS_OK;
}
