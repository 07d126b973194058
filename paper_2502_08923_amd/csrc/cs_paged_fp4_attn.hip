// Attention of a chunk of new rows per stream over the pages of a cache held in 4 bits (Sec. 3.2: the draft
// is appended to the context and evaluated in one pass; App. B.2: per-layer K, V).
//
//   out[r][h] = sum_t p_t v[t] / sum_t p_t,   p_t = exp(scale * q[r][h] . k[t] - max),   t <= L_b + i, t > L_b + i - window
//
// One pass over the tokens with the running maximum and sum of the softmax in float32, as over the wider
// caches, and cut as there (cs_paged_split.h).  Codes become bfloat16 in registers, two an instruction, with
// the scale applied and nothing rounded, and the products are those of the bfloat16 matrix instruction, K as
// the A operand.  Queries and probabilities are NP bfloat16 parts each: one for bfloat16 queries (the
// probabilities are rounded to V's type in the product, half a step of 2^-8), three for float32 queries, which
// hold all 24 bits.  Every sum has one order, given by the cut.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cs_paged_fp4.h"
#include "cs_paged_split.h"

template <int NP>
using f4_qtype = std::conditional_t<NP == 1, bf16_t, float>;

// eight elements at p -> NP parts whose sum they are
__device__ __forceinline__ void f4_split(const bf16_t* p, bf16x8 (&o)[1]) { o[0] = *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ void f4_split8(const float* x, bf16x8 (&o)[3]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bf16_t a = (bf16_t)x[j];
        const float r = x[j] - (float)a;
        const bf16_t b = (bf16_t)r;
        o[0][j] = a;
        o[1][j] = b;
        o[2][j] = (bf16_t)(r - (float)b);
    }
}
__device__ __forceinline__ void f4_split8(const float* x, bf16x8 (&o)[1]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[0][j] = (bf16_t)x[j];
}
__device__ __forceinline__ void f4_split(const float* p, bf16x8 (&o)[3]) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = p[j];
    f4_split8(x, o);
}

// ---- which tiles and tokens a workgroup of the kernel of few rows has ----------------------------------------
// The G * rows query rows of a stream's KV head (row n: block row n / G, head n % G of the group) are cut into
// tiles of TR; streams with qr_lo < G * rows <= qr_hi take part.  W workgroups per KV head are as many as run at
// once, and the tokens are cut among them on the device, from the lengths, by every workgroup for itself:
//   pieces: a workgroup has one piece of one tile, at most `piece` blocks of 32 tokens, with no more than W pieces
//           in all; each lane prices another size, whole tiles among them;
//   shares: the blocks of all tiles are laid end to end and each workgroup takes as many of them: the end of one tile,
//           whole ones, the beginning of another.  For streams of different lengths, where pieces are uneven, and
//           for more tiles than workgroups.
// A cut's price, in blocks of a workgroup that runs alone, is made of its longest workgroup's and of what all tokens cost
// the chip (`bound` times their blocks), as the cube root of their cubes' sum: the larger one, and some more where both
// are alike, for a workgroup is slower among others; and the merge's if there is one.  What a workgroup has of a tile that
// it does not have alone is a partial result, at most two of them, which the merge joins.  (W 0: a workgroup each
// tile, no partial results.)
struct f4_shares {
    int TR, qr_lo, qr_hi;
    int W, least;             // workgroups per KV head; fewest blocks of a piece or a share
    int step;                 // distance of the numbers of pieces tried (W 0: workgroups per KV head)
    float bound, join;        // what a block of all tokens costs the chip, and a merge, in blocks of a workgroup
    int near;                 // neighbouring KV heads that run on one die
    int most;                 // units of all tiles that ascending row offsets can lead to
    float* po;                // [2 W][KVH][TR][hd] partial outputs; 2w: of a tile that an earlier workgroup has begun, 2w + 1: of one that w begins
    float2* pml;              // [2 W][KVH][TR] their (maximum, sum)
    int4* who;                // [2 W] (first row, first query row, query rows, number | workgroups of the tile << 16) for the merge; 0: nothing
};
struct f4_call {
    cs_fp4_dev F;
    pa_args A;
    f4_shares S;
};
__device__ __forceinline__ float f4_price(float longest, float chip) {
    return __builtin_amdgcn_exp2f(__builtin_amdgcn_logf(longest * longest * longest + chip * chip * chip) * (1.0f / 3));
}
struct f4_segment {
    int b, n0;                // stream, first query row
    int off, n;               // first block of the tile's, blocks (W 0: all of them)
    bool first, whole;        // the tile's first blocks, all of its blocks
    int row0, rows, len;      // of the stream
    int number, of;           // of the workgroups that have a part of the tile
};

// A segment costs its start and its end beside its blocks, in blocks of 32 tokens.
#define F4_SEGMENT 10

// tiles of a stream and the blocks that one of them walks (W 0: 1)
__device__ __forceinline__ int2 f4_extent(const cs_pages_dev& D, int G, int window, const f4_shares& S, int rows, int len) {
    const int64_t qr = (int64_t)rows * G;
    if (qr <= S.qr_lo || qr > S.qr_hi) return make_int2(0, 0);
    int span = min(len + rows, D.cap);
    if (window) span = (int)min((int64_t)span, (int64_t)window + min(rows, S.TR / G + 1) + 32);
    return make_int2((int)((qr + S.TR - 1) / S.TR), S.W ? max((span + 31) >> 5, 1) : 1);
}

// Positions count units: blocks of all tiles (shares) or pieces; a lane looks at one of 64 streams.  Units that ascending row
// offsets lead to are at most `most`, which the host keeps below 2^29.  Others may claim rows many times over: sums of units
// stay at 2^30 then, and streams whose sum passes `most` have no work, so that no position ever wraps.
#define F4_MANY (1 << 30)
__device__ __forceinline__ int f4_add(int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)F4_MANY); }
struct f4_walk {
    int p, end;               // position and end of the workgroup's share
    int share;                // units of a share (pieces: 1)
    int piece;                // blocks of a unit (shares: 1)
    int start;                // units that stand for the start of a tile, before its blocks (pieces: 0)
    int b0, before;           // the streams that are looked at, units before them
    int2 e, rows;             // a lane's: tiles, blocks of each; first row and rows
    int len;                  // its length
    int units, upto;          // a lane's: units of a tile; of these streams up to and with its own
    bool have;
};
template <bool ANY>                       // whatever the row offsets are
__device__ __forceinline__ void f4_look_at(const cs_pages_dev& D, int G, int window, const f4_shares& S, f4_walk& k, int lane) {
    k.e = k.rows = make_int2(0, 0), k.len = 0;
    if (k.b0 + lane < D.p.batch) {
        k.rows = cs_stream_rows(D, k.b0 + lane);
        k.len = cs_stream_len(D, k.b0 + lane);
        k.e = f4_extent(D, G, window, S, k.rows.y, k.len);
    }
    k.units = (k.e.y + k.start + k.piece - 1) / k.piece;
    // (a product below 2^30 in float32 is below 2^30 + 2^7)
    if constexpr (ANY) k.upto = pa_wave_reduce((float)k.e.x * (float)k.units < (float)F4_MANY ? k.e.x * k.units : F4_MANY, 0, f4_add);
    else k.upto = pa_wave_scan(k.e.x * k.units);
    k.have = true;
}
__device__ __forceinline__ f4_walk f4_start(const cs_pages_dev& D, int G, int window, const f4_shares& S, int w, int lane) {
    f4_walk k;
    k.p = w, k.end = w + 1, k.share = k.piece = 1, k.start = k.b0 = k.before = 0, k.have = false;
    k.e = k.rows = make_int2(0, 0), k.len = k.units = k.upto = 0;
    const int B = D.p.batch;
    if (!S.W) {
        // The workgroup's stream (b0) and tile (before).  Equal rows: by division.  Streams of at most one tile: one each.  Else
        // stream b has the workgroups from row0[b] * G / TR + b on, which are at least as many as its tiles, and is searched
        // for, 64 places at a time.
        if (!D.row0) {
            const int tiles = max(f4_extent(D, G, window, S, D.rows, 0).x, 1);
            k.b0 = __builtin_amdgcn_readfirstlane(w / tiles);
            k.before = w - k.b0 * tiles;
        } else if (S.qr_hi <= S.TR) k.b0 = w;
        else {
            auto from = [&](int b) { return (int)((int64_t)cs_stream_rows(D, b).x * G / S.TR) + b; };
            int lo = 0, n = B;
            while (n > 1) {
                const int step = (n + 63) >> 6, b = lo + lane * step;
                const int c = __popcll(__ballot(b < lo + n && from(min(b, B - 1)) <= w));
                const int skip = max(c - 1, 0) * step;
                lo += skip;
                n = min(n - skip, step);
            }
            k.b0 = lo;
            k.before = w - __builtin_amdgcn_readfirstlane(from(lo));
        }
        if (k.b0 >= B || k.before < 0) k.end = k.p;
        return k;
    }
    int all = 0, tiles = 0;
    k.start = F4_SEGMENT;
    for (; k.b0 < B; k.b0 += 64) {
        f4_look_at<true>(D, G, window, S, k, lane);
        all = f4_add(all, __builtin_amdgcn_readlane(k.upto, 63));
        if (B <= 64) {
            tiles = __builtin_amdgcn_readlane(pa_wave_scan(k.e.x), 63);
            break;
        }
    }
    if (all > S.most) all = 0, tiles = S.W + 1;                 // (row offsets that make no sense: nothing to share out)
    k.share = max((all + S.W - 1) / S.W, S.least);
    if (B <= 64 && tiles <= S.W) {
        const int longest = __builtin_amdgcn_readlane(pa_wave_reduce(k.e.y, 0, [](int a, int b) { return max(a, b); }), 63);
        const int n = 1 + lane * S.step, cut = max((longest + n - 1) / n, S.least);
        const float inv = 1.0f / (float)cut;
        int count = 0;
        for (int i = 0; i < B; ++i) {
            const int blocks = __builtin_amdgcn_readlane(k.e.y, i), q = (int)((float)blocks * inv), r = blocks - q * cut;
            count += __builtin_amdgcn_readlane(k.e.x, i) * (q + (r > 0) + (r > cut));             // (q is off by one at most)
        }
        const float least = (float)(all - F4_SEGMENT * tiles) * S.bound;
        const float cost = f4_price((float)cut, least) + (cut < longest ? S.join + (float)n * 0.1f : 0.f);
        // (costs are positive: their bits are ordered as they are)
        const int bits = count <= S.W ? __float_as_int(cost) : 0x7f800000;
        const int best = __builtin_amdgcn_readlane(pa_wave_reduce(bits, 0x7f800000, [](int a, int b) { return min(a, b); }), 63);
        if (__int_as_float(best) <= f4_price((float)(k.share + F4_SEGMENT), least) + S.join) {
            k.piece = __builtin_amdgcn_readlane(cut, __ffsll(__ballot(bits == best)) - 1);
            k.share = 1;
            k.start = 0;
            k.units = (k.e.y + k.piece - 1) / k.piece;
            k.upto = pa_wave_scan(k.e.x * k.units);
            all = __builtin_amdgcn_readlane(k.upto, 63);
        }
    }
    k.b0 = 0;
    k.have = B <= 64;
    k.p = (int)min((int64_t)k.share * w, (int64_t)all);
    k.end = min(k.p + k.share, all);
    return k;
}
__device__ __forceinline__ bool f4_next(const cs_pages_dev& D, int G, int window, const f4_shares& S, int w, f4_walk& k, int lane, f4_segment& o) {
    if (k.p >= k.end) return false;
    if (!S.W) {
        k.p = k.end;
        const int2 rows = cs_stream_rows(D, k.b0);
        o.b = k.b0;
        o.row0 = __builtin_amdgcn_readfirstlane(rows.x), o.rows = __builtin_amdgcn_readfirstlane(rows.y);
        o.len = __builtin_amdgcn_readfirstlane(cs_stream_len(D, k.b0));
        o.n0 = k.before * S.TR;
        o.off = 0, o.n = 1;
        o.first = o.whole = true;
        o.number = 0, o.of = 1;
        return k.before < f4_extent(D, G, window, S, o.rows, o.len).x;
    }
    for (;;) {
        if (!k.have) f4_look_at<false>(D, G, window, S, k, lane);
        const int all = __builtin_amdgcn_readlane(k.upto, 63);
        if (k.p < k.before + all) break;
        k.before += all;
        k.b0 += 64;
        k.have = false;
        if (k.b0 >= D.p.batch) return false;                    // (more workgroups than tiles)
    }
    const unsigned long long past = __ballot(k.before + k.upto > k.p);
    if (!past) return false;                                    // (offsets or lengths that change while the call runs)
    const int l = __ffsll(past) - 1;
    const int tiles = __builtin_amdgcn_readlane(k.e.x, l), blocks = __builtin_amdgcn_readlane(k.e.y, l), units = __builtin_amdgcn_readlane(k.units, l);
    o.row0 = __builtin_amdgcn_readlane(k.rows.x, l), o.rows = __builtin_amdgcn_readlane(k.rows.y, l), o.len = __builtin_amdgcn_readlane(k.len, l);
    const unsigned at = k.p - (k.before + __builtin_amdgcn_readlane(k.upto, l) - tiles * units);
    const int tile = __builtin_amdgcn_readfirstlane(tiles == 1 ? 0 : at / (unsigned)units), off = at - tile * units;
    if ((unsigned)tile >= (unsigned)tiles) return false;        // (as above)
    const int n = min(units - off, k.end - k.p);
    o.b = k.b0 + l;
    o.n0 = tile * S.TR;
    o.off = max(off * k.piece - k.start, 0);
    o.n = max((off + n) * k.piece - k.start, 0) - o.off;
    o.first = off == 0;
    o.whole = n == units;
    o.number = 0, o.of = 1;
    if (!o.whole) {
        const int first = __builtin_amdgcn_readfirstlane((unsigned)(k.p - off) / (unsigned)k.share);
        o.number = w - first;
        o.of = __builtin_amdgcn_readfirstlane((unsigned)(k.p - off + units - 1) / (unsigned)k.share) - first + 1;
    }
    k.p += n;
    return true;
}
// Workgroup -> (w, KV head).  Dies take workgroups in turn, eight of them, each with a cache of its own: `near` heads whose
// rows share cache lines (a token-major pool has 64 bytes of codes of a head of 128 features next to its neighbour's)
// are eight workgroups apart.
__device__ __forceinline__ int2 f4_whose(unsigned wg, int KVH, int W_all, int near) {
    const int groups = KVH / near, whole = W_all * groups >> 3;              // (w, head group) pairs, in eights
    const int i = wg >> 3, x = wg & 7, turn = i / near;
    int u, j;
    if (turn < whole) u = turn * 8 + x, j = i - turn * near;
    else {
        const int r = wg - whole * 8 * near;
        u = whole * 8 + r / near, j = r % near;
    }
    const int w = u / groups;
    return make_int2(w, (u - w * groups) * near + j);
}

// ---- few query rows: the stream of codes is the bound ---------------------------------------------------
// Four waves share a tile of up to 48 query rows and take the 32-token blocks of a token range in turn; codes,
// scores and outputs stay in registers:
//   S^T[token][row] = K . Q^T           A = 16 key rows, B = query rows
//   O^T[feature][row] += V^T . P^T      A = 16 features of 32 tokens, B = the probabilities as S^T left them
// Which token is which row of A, and which feature which k of the first product, is free as long as both
// operands agree.  Lane (c, g) takes the features g * HD / 4 .. of its key rows, which is 16 bytes of codes
// under one scale at HD = 128, and row c of half a is token 8 (c / 4) + 4 a + c % 4 of the block, so that the
// rows of S^T that the lane gets, and the value rows it needs, are the tokens 8g .. 8g + 7: their scales are
// eight bytes of the page.  Of those value rows a lane loads HD / 16 features each, makes them bfloat16 and
// turns pairs of tokens with byte permutes into the A fragments: fragment u has feature c * HD / 16 + u in row
// c.  A page holds whole blocks, so every load has one page, a uniform base, and nothing to check.
//
// Single tokens are bound by memory: 64 streams of 8191 tokens, 8 heads of 128, 108 us = 5.3 TB/s of codes and scales; 64 of 2 to 8
// thousand over token-major pages of 32, where a head's codes are half lines, 94 us = 3.8 TB/s with 1.03 times the bytes read (tried at
// earlier states: two heads in one workgroup 149 us against 138 on one die; in one wave 98 against 97; four or all eight on one die no
// change).  48 rows: 8 x 11 rows behind 18431 51 to 54 us a captured call, 48 for the kernel and 6 for the join under the profiler.  Neither
// unit is full (vector 60 %, matrix 30 % busy); a block is 64 conversions, 32 permutes, 24 exponentials and 51 products a wave, two waves
// a SIMD, and about 14 us do not grow with the context: launches, the look-up of the cut, the exchange, the join.
// Two workgroups a compute unit: with registers for three 48 rows take 93 us for 51, for one 75 (single tokens over token-major
// pages 127 and 86 for 94, of 256 features 124 and 50 for 45, of 64 features 45 and 47 for 47).  Of 256 features and one part 9 registers
// spill, of 48 float32 rows and 128 features 7.  (Queries in registers and 64 tokens a softmax step, tried at an earlier state: 100 us for
// 57, no gain.)
#define F4N_WAVES 4
template <int HD>
struct f4_keys { u32x4 k[2][HD == 256 ? 2 : 1]; u32x2 s[HD == 256 ? 2 : 1]; };
template <int HD>
struct f4_values { unsigned v[8][HD == 256 ? 2 : 1]; u32x2 s; };

template <int HD, int NT, int NP, bool KLDS>
__global__ __launch_bounds__(64 * F4N_WAVES, 2) void k_paged_fp4_narrow(f4_call C) {
    typedef f4_qtype<NP> T_;
    constexpr int KS = HD / 32, MT = HD / 16, VF = HD / 16;
    constexpr int KB = HD == 256 ? 2 : 1;                       // 32-feature pieces of a lane's key row (HD 64: half of one)
    constexpr int VW = HD == 256 ? 2 : 1;                       // dwords of a lane's value row (HD 64: half of one)
    constexpr bool QREG = NT == 1 && NP == 1;                   // the query fragments stay in registers, else they are read from LDS
    // blocks in flight (captured calls.  One more: 48 rows 59 us for 51, single tokens of 256 features 67 for 45, which spill more,
    // of 128 features 96 for 94.  One less: of 256 features 42.5 for 45, 16 rows 47 for 51 and in float32 50 for 53; others within 2 %)
    constexpr int AHEAD = NT > 1 ? 1 : HD == 256 || NP > 1 ? 2 : 3;
    constexpr int ROWS = 16 * NT, QROW = HD * 2 + 16, QPLANE = ROWS * QROW;
    constexpr int SLOT = NT * (2 * VF / 4 * 1024 + 512);        // half of a wave's O, with its maximum and sum
    constexpr int LDS_BYTES = F4N_WAVES * SLOT > NP * QPLANE ? F4N_WAVES * SLOT : NP * QPLANE;
    static_assert(F4N_WAVES == 4, "two exchanges");
    __shared__ __attribute__((aligned(16))) unsigned char smem[LDS_BYTES];
    // KLDS, where key rows lie apart: sixteen of them are requested with four neighbouring lanes on the 64 bytes of each, so that
    // neighbours share lines, and go to the lanes that multiply them through LDS of the wave's own.  (Requested by those
    // lanes themselves: 64 single tokens of 2 to 8 thousand over token-major pages 97.4 us for 94.1, 1024 of 100 100 for 95;
    // head-major pages 1 % slower, more rows and the values the same way no change.)
    static_assert(!KLDS || HD == 128, "a lane's key row is one load");
    constexpr int KROW = HD / 2 + 16, KTILE = 16 * KROW;
    __shared__ __attribute__((aligned(16))) unsigned char kmem[KLDS ? F4N_WAVES * 2 * KTILE : 16];
    // The arguments fill the scalar registers several times over.  Read anew for every segment and behind its loop, they
    // are not carried through it.
    typedef const __attribute__((address_space(4))) f4_call* call_ptr;
    auto call = [&]() -> const f4_call& {
        call_ptr p = (call_ptr)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(p));
        return *(const f4_call*)p;
    };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    int w, kvh;
    f4_walk walk;
    {
        const f4_call& C0 = call();
        const int2 o = f4_whose(cs_paged_wg(), C0.F.d.p.n_kv_heads, C0.S.W ? C0.S.W : C0.S.step, C0.S.near);
        w = __builtin_amdgcn_readfirstlane(o.x), kvh = __builtin_amdgcn_readfirstlane(o.y);
        walk = f4_start(C0.F.d, C0.A.G, C0.A.window, C0.S, w, lane);
        if (C0.S.W && kvh == 0 && tid == 0) C0.S.who[2 * w] = C0.S.who[2 * w + 1] = make_int4(0, 0, 0, 0);
    }
    f4_segment K;
    for (;;) {
    const f4_call& C1 = call();
    const cs_fp4_dev& F = C1.F;
    const cs_pages_dev& D = F.d;
    const pa_args& A = C1.A;
    if (!f4_next(D, A.G, A.window, C1.S, w, walk, lane, K)) return;
    if (NT > 1 || HD == 256) walk.have = false;         // (registers: the streams are looked at again)
    const int hd = D.p.head_dim, cap = D.cap;
    pa_tile T;
    T.b = K.b;
    T.n0 = K.n0;
    T.row0 = K.row0;
    T.rows = K.rows;
    T.QR = T.rows * A.G;
    T.L = K.len;
    if (!QREG) __syncthreads();                         // every wave is done with the segment before
    const int n_rows = min(ROWS, T.QR - T.n0);          // live query rows of the tile
    const int i_lo = T.n0 / A.G, i_hi = (T.n0 + n_rows - 1) / A.G;
    const int n_tok = min(T.L + i_hi + 1, D.cap);       // tokens that the tile's last row sees
    const int base = A.window ? max(0, T.L + i_lo - A.window + 1) & ~31 : 0;
    const int w_begin = (int)min((int64_t)base + (int64_t)K.off * 32, (int64_t)n_tok);
    const int t_end = K.number == K.of - 1 ? n_tok : (int)min((int64_t)base + ((int64_t)K.off + K.n) * 32, (int64_t)n_tok);
    // blocks between these need no mask
    const int open_lo = A.window ? T.L + i_hi - A.window + 1 : 0, open_hi = min(T.L + i_lo + 1, D.cap);
    const int w_first = A.window ? T.L + i_lo - A.window + 1 : 0;       // tokens before it are seen by no row of the tile

    const int32_t* tab = D.p.table + T.b * D.p.table_stride;
    constexpr int STEP = 32 * F4N_WAVES;
    // the page of the lane's first block: on its way while the query rows are
    int page_next = 0;
    if (w_begin + 32 * wave < t_end) page_next = tab[min(w_begin + 32 * wave + lane * STEP, (t_end - 1) & ~31) >> D.page_log2];

    bf16x8 qreg[KS];
    if constexpr (QREG) {
        const int i = (T.n0 + c) / A.G, h = kvh * A.G + T.n0 + c - i * A.G;
        const bf16_t* qp = (const bf16_t*)A.q + (T.row0 + i) * A.q_row + h * A.q_head + g * (HD / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qreg[s] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (c < n_rows && g * (HD / 4) + s * 8 < hd) qreg[s] = *reinterpret_cast<const bf16x8*>(qp + s * 8);
        }
    } else {
        // query rows into LDS, all loads before the first store
        constexpr int EACH = (ROWS * (HD / 8) + 64 * F4N_WAVES - 1) / (64 * F4N_WAVES);
        bf16x8 v[EACH][NP];
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            const int idx = tid + x * 64 * F4N_WAVES, n = idx / (HD / 8), seg = idx % (HD / 8);
#pragma unroll
            for (int p = 0; p < NP; ++p) v[x][p] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (n < n_rows && seg * 8 < hd) {
                const int i = (T.n0 + n) / A.G, h = kvh * A.G + T.n0 + n - i * A.G;
                f4_split((const T_*)A.q + (T.row0 + i) * A.q_row + h * A.q_head + seg * 8, v[x]);
            }
        }
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            const int idx = tid + x * 64 * F4N_WAVES, n = idx / (HD / 8), seg = idx % (HD / 8);
            if (n < ROWS)
#pragma unroll
                for (int p = 0; p < NP; ++p) *reinterpret_cast<bf16x8*>(smem + p * QPLANE + n * QROW + seg * 16) = v[x][p];
        }
    }
    int q_last[NT];                                     // the last token that the lane's query rows see, and how many before it
    const int back = A.window ? A.window - 1 : 0x3fffffff;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = nt * 16 + c;
        q_last[nt] = n < n_rows ? T.L + (T.n0 + n) / A.G : -1;
    }

    const uint8_t *Kh = F.k + kvh * F.k_head, *Vh = F.v + kvh * F.v_head, *KSh = F.ks + kvh * F.ks_head, *VSh = F.vs + kvh * F.vs_head;
    // (features that the head does not have are read at feature 0: their query elements are 0, their outputs are not stored)
    unsigned koff[KB], ksoff[KB], voff, vsoff;
    const unsigned kts = (unsigned)F.k_token, vts = (unsigned)F.v_token;
    {
#pragma unroll
        for (int h = 0; h < KB; ++h) {
            const int f = g * (HD / 4) + h * 32 < hd ? g * (HD / 4) + h * 32 : 0;
            koff[h] = (8 * (c >> 2) + (c & 3)) * kts + f / 2;
            if (KLDS) {
                const int r = lane >> 2, fr = (lane & 3) * 32 < hd ? (lane & 3) * 32 : 0;
                koff[h] = (8 * (r >> 2) + (r & 3)) * kts + fr / 2;
            }
            ksoff[h] = f / CS_FP4_GROUP * (unsigned)F.ks_group + 8 * (c >> 2);
        }
        const int f = c * VF < hd ? c * VF : 0;
        voff = 8 * g * vts + f / 2;
        vsoff = f / CS_FP4_GROUP * (unsigned)F.vs_group + 8 * g;
    }

    f32x4 oacc[MT][NT], lacc[NT];
    float m_run[NT], thr[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = thr[nt] = -INFINITY;
        lacc[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) oacc[mt][nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const bf16_t one = (bf16_t)1.0f;
    const bf16x8 ones = (bf16x8){one, one, one, one, one, one, one, one};
    const float scale2 = A.scale2, inv_scale2 = 1.0f / A.scale2;
    const int kshift = 8 * (c & 3);
    if (!QREG) __syncthreads();

    // A lane holds one of the wave's next 64 blocks: where in the pools it starts, so that a request costs the scalar
    // unit no multiplications.  A block whose page does not exist is read from page 0 and masked; a lane that has none
    // repeats the wave's last one.
    for (int seg0 = w_begin; seg0 < t_end; seg0 += 64 * STEP) {
        const int t_begin = seg0 + 32 * wave;
        const int n_all = t_begin < t_end ? min(64, (t_end - t_begin + STEP - 1) / STEP) : 0;
        if (n_all == 0) continue;
        uint64_t at_k, at_v, at_ks, at_vs;
        unsigned long long okay;
        {
            const int tb = t_begin + min(lane, n_all - 1) * STEP, slot = tb & (D.p.page_size - 1);
            const int page = seg0 == w_begin ? page_next : tab[tb >> D.page_log2];
            const bool ok = (unsigned)page < (unsigned)D.p.n_pages;
            const int64_t pg = ok ? page : 0;
            okay = __ballot(ok);
            at_k = (uint64_t)(Kh + pg * F.k_page + slot * F.k_token);
            at_v = (uint64_t)(Vh + pg * F.v_page + slot * F.v_token);
            at_ks = (uint64_t)(KSh + pg * F.ks_page + slot);
            at_vs = (uint64_t)(VSh + pg * F.vs_page + slot);
        }
        auto at = [&](int i) { return t_begin + i * STEP; };
        auto from = [&](uint64_t a, int i) {
            return cs_rsrc((const void*)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(a >> 32), i & 63) << 32 |
                                         (unsigned)__builtin_amdgcn_readlane((int)a, i & 63)), 0x80000000u);
        };
        auto ldk = [&](f4_keys<HD>& b, int i) {
            const auto p = from(at_k, i), f = from(at_ks, i);
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int h = 0; h < KB; ++h) {
                    if constexpr (HD == 64) {
                        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(p, koff[h], a * 4 * kts, 0));
                        b.k[a][h][0] = x[0];
                        b.k[a][h][1] = x[1];
                    } else b.k[a][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, koff[h], a * 4 * kts, 0));
                }
#pragma unroll
            for (int h = 0; h < KB; ++h) b.s[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(f, ksoff[h], 0, 0));
        };
        auto ldv = [&](f4_values<HD>& b, int i) {
            const auto p = from(at_v, i), f = from(at_vs, i);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (HD == 64) b.v[e][0] = __builtin_amdgcn_raw_buffer_load_b16(p, voff, e * vts, 0);
                else if constexpr (HD == 128) b.v[e][0] = __builtin_amdgcn_raw_buffer_load_b32(p, voff, e * vts, 0);
                else {
                    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(p, voff, e * vts, 0));
                    b.v[e][0] = x[0];
                    b.v[e][VW - 1] = x[1];
                }
            }
            b.s = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(f, vsoff, 0, 0));
        };
        auto block = [&](f4_keys<HD>& kb, f4_values<HD>& vb, int i) {
            f32x4 sacc[2][NT];
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) sacc[a][nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if constexpr (KLDS) {
                unsigned char* t = kmem + wave * 2 * KTILE;
#pragma unroll
                for (int a = 0; a < 2; ++a) *reinterpret_cast<u32x4*>(t + a * KTILE + (lane >> 2) * KROW + (lane & 3) * 16) = kb.k[a][0];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
                for (int a = 0; a < 2; ++a) kb.k[a][0] = *reinterpret_cast<const u32x4*>(t + a * KTILE + c * KROW + g * 16);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int h = s / 4, d = s % 4;
                bf16x8 kf[2];
#pragma unroll
                for (int a = 0; a < 2; ++a) kf[a] = cs_fp4_decode(kb.k[a][h][d], kb.s[h][a] >> kshift << 23);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        const bf16x8 qb = QREG ? qreg[s] : *reinterpret_cast<const bf16x8*>(smem + p * QPLANE + (nt * 16 + c) * QROW + g * (HD / 2) + s * 16);
#pragma unroll
                        for (int a = 0; a < 2; ++a) sacc[a][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[a], qb, sacc[a][nt], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            ldk(kb, i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = at(i);
            const bool gone = !(okay >> i & 1), masked = t0 < open_lo || t0 + 32 > open_hi || gone;
            if (masked) {
                const int t = t0 + 8 * g;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool sees = t + e <= q_last[nt] && t + e >= q_last[nt] - back && t + e < cap && !gone;
                        sacc[e >> 2][nt][e & 3] = sees ? sacc[e >> 2][nt][e & 3] : -INFINITY;
                    }
                // what lies behind the last token, in place of a page or before every window may have any scale, and 0 *
                // anything must stay 0: with scale byte 0 every code is finite
                const int e0 = min(max(w_first - t, 0), 8), e1 = gone ? 0 : min(max(n_tok - t, 0), 8);
                const uint64_t from = e0 < 8 ? ~(uint64_t)0 << 8 * e0 : 0, to = e1 < 8 ? ~(~(uint64_t)0 << 8 * e1) : ~(uint64_t)0;
                vb.s[0] &= (unsigned)(from & to);
                vb.s[1] &= (unsigned)((from & to) >> 32);
            }
            // the reference maximum of a row moves (and O is rescaled) only when it is left behind by 2^8
            bool over = masked;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float lm = -INFINITY;
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) lm = fmaxf(lm, sacc[a][nt][j]);
                over |= !(lm <= thr[nt]);
            }
            if (__any(over)) {
                bool moved = false;
                float alpha[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sacc[a][nt][j]);
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
            }
            bf16x8 pb[NT][NP];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m_safe = m_run[nt] == -INFINITY ? 0.f : m_run[nt];
                float sv[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) sv[e] = __builtin_amdgcn_exp2f(fmaf(sacc[e >> 2][nt][e & 3], scale2, -m_safe));
                f4_split8(sv, pb[nt]);
            }
            // (the row sum is that of the rounded probabilities)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int p = 0; p < NP; ++p) lacc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[nt][p], lacc[nt], 0, 0, 0);
            // two features of the lane at a time: byte d of its eight value rows
#pragma unroll
            for (int d = 0; d < VF / 2; ++d) {
                unsigned w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned x = vb.v[e][d / 4];
                    const float s = __uint_as_float(vb.s[e >> 2] >> 8 * (e & 3) << 23);
                    bf16x2 r;
                    if (d % 4 == 0) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 0);
                    else if (d % 4 == 1) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 1);
                    else if (d % 4 == 2) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 2);
                    else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 3);
                    w[e] = __builtin_bit_cast(unsigned, r);
                }
                u32x4 lo, hi;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    lo[r] = __builtin_amdgcn_perm(w[2 * r + 1], w[2 * r], 0x05040100u);
                    hi[r] = __builtin_amdgcn_perm(w[2 * r + 1], w[2 * r], 0x07060302u);
                }
                const bf16x8 fl = __builtin_bit_cast(bf16x8, lo), fh = __builtin_bit_cast(bf16x8, hi);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        oacc[2 * d][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fl, pb[nt][p], oacc[2 * d][nt], 0, 0, 0);
                        oacc[2 * d + 1][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh, pb[nt][p], oacc[2 * d + 1][nt], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            ldv(vb, i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        };
        f4_keys<HD> kb[AHEAD];
        f4_values<HD> vb[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            ldk(kb[j], j);
            __builtin_amdgcn_sched_barrier(0);
            ldv(vb[j], j);
        }
        int i = 0;
        for (; i + AHEAD <= n_all; i += AHEAD) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) block(kb[j], vb[j], i + j);
        }
#pragma unroll
        for (int j = 0; j < AHEAD - 1; ++j)
            if (i + j < n_all) block(kb[j], vb[j], i + j);
    }

    // The waves' (maximum, sum, O) are joined in two exchanges, first with the wave two away, then with the neighbour, of
    // half of what there is each time, so that wave w ends with element j = w of every accumulator.  oacc[u][nt][j]:
    // query row nt*16 + c, feature (4g + j) * VF + u
    float l_run[NT], mine2[MT][NT][2], mine1[MT][NT];
    auto swap = [&](int partner, auto send, auto keep, auto n_tag) {
        constexpr int N = decltype(n_tag)::value;               // elements of an accumulator that are sent, and kept
        __syncthreads();             // (first: every wave is done with the query rows, or the exchange before)
        unsigned char* to = smem + partner * SLOT;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int u = 0; u < VF; u += 4)
                    *reinterpret_cast<f32x4*>(to + (((nt * N + j) * (VF / 4) + u / 4) * 64 + lane) * 16) =
                        (f32x4){send(u, nt, j), send(u + 1, nt, j), send(u + 2, nt, j), send(u + 3, nt, j)};
            *reinterpret_cast<float2*>(to + SLOT - NT * 512 + (nt * 64 + lane) * 8) = make_float2(m_run[nt], l_run[nt]);
        }
        __syncthreads();
        const unsigned char* from = smem + wave * SLOT;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float2 ml = *reinterpret_cast<const float2*>(from + SLOT - NT * 512 + (nt * 64 + lane) * 8);
            const float M = fmaxf(m_run[nt], ml.x), Ms = M == -INFINITY ? 0.f : M;
            const float f0 = __builtin_amdgcn_exp2f(m_run[nt] - Ms), f1 = __builtin_amdgcn_exp2f(ml.x - Ms);
            m_run[nt] = M;
            l_run[nt] = f0 * l_run[nt] + f1 * ml.y;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int u = 0; u < VF; u += 4) {
                    const f32x4 o = *reinterpret_cast<const f32x4*>(from + (((nt * N + j) * (VF / 4) + u / 4) * 64 + lane) * 16);
#pragma unroll
                    for (int x = 0; x < 4; ++x) keep(u + x, nt, j, f0, f1 * o[x]);
                }
        }
    };
    // (by masks: a choice between two elements of an accumulator becomes an index into it, which registers do not have)
    const unsigned high = wave >= 2 ? ~0u : 0u, odd = wave & 1 ? ~0u : 0u;
    auto pick = [](unsigned m, float a, float b) { return __uint_as_float((__float_as_uint(a) & m) | (__float_as_uint(b) & ~m)); };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l_run[nt] = lacc[nt][0];
    swap(wave ^ 2, [&](int u, int nt, int j) { return pick(high, oacc[u][nt][j], oacc[u][nt][2 + j]); },
         [&](int u, int nt, int j, float f, float add) { mine2[u][nt][j] = f * pick(high, oacc[u][nt][2 + j], oacc[u][nt][j]) + add; },
         std::integral_constant<int, 2>());
    swap(wave ^ 1, [&](int u, int nt, int) { return pick(odd, mine2[u][nt][0], mine2[u][nt][1]); },
         [&](int u, int nt, int, float f, float add) { mine1[u][nt] = f * pick(odd, mine2[u][nt][1], mine2[u][nt][0]) + add; },
         std::integral_constant<int, 1>());
    const f4_call& C2 = call();
    const f4_shares& S = C2.S;
    const int part = 2 * w + K.first, KVH = C2.F.d.p.n_kv_heads, j = wave;
    if (!K.whole && kvh == 0 && tid == 0) S.who[part] = make_int4(T.row0, T.n0, T.QR, K.number | K.of << 16);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = nt * 16 + c;
        if (n >= n_rows) continue;
        const int i = (T.n0 + n) / C2.A.G, h = kvh * C2.A.G + T.n0 + n - i * C2.A.G;
        const int64_t r = T.row0 + i, row = ((int64_t)part * KVH + kvh) * S.TR + n;
        const float inv = l_run[nt] > 0.f ? 1.0f / l_run[nt] : 0.f;           // a row that sees nothing: 0
        if (tid < 16 && !K.whole) S.pml[row] = make_float2(m_run[nt], l_run[nt]);
#pragma unroll
        for (int u = 0; u < VF; u += 4) {
            const int d = (4 * g + j) * VF + u;
            const f32x4 o = (f32x4){mine1[u][nt], mine1[u + 1][nt], mine1[u + 2][nt], mine1[u + 3][nt]};
            if (d >= hd) continue;
            if (K.whole) pa_store4((T_*)C2.A.out + r * C2.A.out_row + h * C2.A.out_head + d, o * inv);
            else pa_store4(S.po + row * hd + d, o);
        }
    }
    }
}

// out[r][h] = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the workgroups that have a part of a tile, which share
// out its rows.  Parts are waited for, so a row's are spread over 2^teams_log2 teams of 2^lanes_log2 lanes, four of them a
// team, as far as the workgroup has teams; a lane of a team has four of the hd features, and reads the (maximum,
// sum) pairs of every lanes-th part, whose weights go round by shuffles.  (Eight parts of 8 x 44 rows and 8 heads of 128,
// 11 MB: 6.5 us, a launch's own 3 among them.)
#define F4J_THREADS 256
template <typename T_>
__global__ __launch_bounds__(F4J_THREADS) void k_paged_fp4_join(cs_pages_dev D, pa_args A, f4_shares S, int lanes_log2) {
    __shared__ f32x4 s_acc[F4J_THREADS];
    __shared__ float s_l[F4J_THREADS];
    const int KVH = D.p.n_kv_heads, kvh = blockIdx.x % KVH, w = blockIdx.x / KVH;
    const int lanes = 1 << lanes_log2, sub = threadIdx.x & (lanes - 1), d = sub * 4, hd = D.p.head_dim;
    for (int side = 0; side < 2; ++side) {
        const int4 who = S.who[2 * w + side];
        const int number = who.w & 0xffff, of = who.w >> 16, first = 2 * (w - number);
        if (of <= 1) continue;
        int teams_log2 = 0;
        while (4 << teams_log2 < of && lanes << (teams_log2 + 1) <= F4J_THREADS) ++teams_log2;
        const int teams = 1 << teams_log2, per = F4J_THREADS >> (lanes_log2 + teams_log2), team = threadIdx.x >> lanes_log2 & (teams - 1);
        const int rows = min(S.TR, who.z - who.y);
        for (int n0 = number * per; n0 < rows; n0 += of * per) {
            const int n = n0 + (threadIdx.x >> (lanes_log2 + teams_log2));
            // (part s: the first workgroup's beginning of the tile, then what the others have of one begun before)
            auto at = [&](int s) { return ((int64_t)(first + (s ? 2 * s : 1)) * KVH + kvh) * S.TR + min(n, rows - 1); };
            float M = -INFINITY;
            for (int s = sub; s < of; s += lanes) M = fmaxf(M, S.pml[at(s)].x);
            for (int o = lanes >> 1; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
            const float Ms = M == -INFINITY ? 0.f : M;
            f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
            float l = 0.f;
            for (int s0 = 0; s0 < of; s0 += lanes) {
                float2 ml = make_float2(-INFINITY, 0.f);
                if (s0 + sub < of) ml = S.pml[at(s0 + sub)];
                const float f = __builtin_amdgcn_exp2f(ml.x - Ms), fl = f * ml.y;
                const int ns = min(lanes, of - s0);
                for (int s = team; s < ns; s += 4 * teams)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        // (past the last part: weight 0, its row once more; one that saw nothing has stored zeros)
                        const int m = min(s + u * teams, ns - 1), from = (threadIdx.x & 63 & ~(lanes - 1)) + m;
                        const float keep = s + u * teams < ns ? 1.f : 0.f;
                        l += keep * __shfl(fl, from, 64);
                        acc += keep * __shfl(f, from, 64) * *reinterpret_cast<const f32x4*>(S.po + at(s0 + m) * hd + min(d, hd - 4));
                    }
            }
            if (teams > 1) {
                __syncthreads();
                s_acc[threadIdx.x] = acc;
                s_l[threadIdx.x] = l;
                __syncthreads();
                if (team) continue;
                for (int i = 1; i < teams; ++i) {
                    acc += s_acc[threadIdx.x + i * lanes];
                    l += s_l[threadIdx.x + i * lanes];
                }
            }
            const int i = (who.y + n) / A.G, h = kvh * A.G + who.y + n - i * A.G;
            if (n < rows && d < hd) pa_store4((T_*)A.out + (int64_t)(who.x + i) * A.out_row + h * A.out_head + d, acc * (l > 0.f ? 1.0f / l : 0.f));
        }
    }
}

// ---- many query rows: the matrix cores and the vector unit are the bound --------------------------------
// Eight waves have 16 * NT query rows each and walk the tokens together, 64 at a time.  Codes are made
// bfloat16 once for all of them: every wave takes eight of the next 64 tokens' key and value rows from registers,
// where their codes have arrived meanwhile, and lays them down in the other half of LDS while the waves
// multiply out of this one.
//   keys: 16 tokens x 32 features in fragment order, a lane's 16 bytes are what it multiplies
//   values: 16 tokens x 32 features as two 16 x 16 squares of 32-byte rows for the transposing LDS read
// What is dead or behind every window is laid down under scale byte 0, finite whatever it is, so only the scores
// have a mask.
//
// 16 x 33 rows of 28 heads behind 65535: 498 us a call = 1.0 PFLOP/s; 4096 rows on an empty cache 145 us = 0.95; 2048 rows behind 16384
// 1.05 (an 8192^3 library product: 1.22).  Matrix and vector unit are each busy half of the time and overlap little.  64 tokens a
// softmax step instead of 32: 578 -> 497 us.  Tried against that: the waves of a SIMD at different points of the
// loop with a third stage in LDS (1 to 3 % slower), priorities fixed by wave (2 to 8 %) or none (1 to 2 %), laying down after the scores (4 %) or
// skewed between the halves of the workgroup (15 %).
#define F4W_WAVES 8
template <int HD, int NT, int NP>
__global__ __launch_bounds__(64 * F4W_WAVES) void k_paged_fp4_wide(cs_fp4_dev F, pa_args A, pa_plan P) {
    typedef f4_qtype<NP> T_;
    constexpr int KS = HD / 32, MT = HD / 16;
    constexpr int WROWS = 16 * NT, TR = F4W_WAVES * WROWS;
    constexpr int NB = HD <= 128 || NP == 1 ? 2 : 1;             // blocks of 32 tokens that go through the softmax together
    constexpr int DW = HD / 64;                                 // dwords of codes of a lane's piece of a row
    constexpr int HALF = 2 * KS * 1024, V_AT = 2 * HALF, STAGE_BYTES = 2 * V_AT;         // keys of a block; of a stage
    __shared__ __attribute__((aligned(16))) unsigned char stage[2][STAGE_BYTES];
    const cs_pages_dev& D = F.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int KVH = D.p.n_kv_heads;
    const unsigned wg = cs_paged_wg();
    const int kvh = wg % KVH;
    pa_work K;
    if (!pa_find(D, A.G, A.window, P, wg / KVH, kvh, K)) return;
    const pa_tile& T = K.T;
    const int hd = D.p.head_dim, G = A.G;
    const int n_rows = min(TR, T.QR - T.n0);
    const int i_lo = T.n0 / G, i_hi = (T.n0 + n_rows - 1) / G;
    const int n_lim = min(T.L + i_hi + 1, D.cap);              // tokens that the tile's last row sees
    const int w_first = A.window ? T.L + i_lo - A.window + 1 : 0;       // tokens before it are seen by no row of the tile
    const int base = A.window ? max(0, w_first) & ~31 : 0;
    const int w_begin = (int)min((int64_t)base + (int64_t)K.split * K.chunk, (int64_t)n_lim);
    const int t_end = K.split == K.nsplit - 1 ? n_lim : (int)min((int64_t)w_begin + K.chunk, (int64_t)n_lim);
    const int n_stages = (t_end - w_begin + 63) / 64;

    const int n0 = T.n0 + wave * WROWS + c;
    bf16x8 qreg[NT][KS][NP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = n0 + nt * 16, i = n / G;
        const T_* qp = (const T_*)A.q + (T.row0 + i) * A.q_row + (kvh * G + n - i * G) * A.q_head + g * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int p = 0; p < NP; ++p) qreg[nt][s][p] = (bf16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (n < T.QR && s * 32 < hd) f4_split(qp + s * 32, qreg[nt][s]);
        }
    }

    // a lane's piece of the 64 tokens: features (lane / 8) * HD / 8 .. of token 8 * wave + lane % 8
    const int tok = 8 * wave + (lane & 7), f0 = (lane >> 3) * (HD / 8);
    const bool there = f0 < hd;
    constexpr unsigned NOWHERE = 0x80000000u;
    const unsigned kts = (unsigned)F.k_token, vts = (unsigned)F.v_token, kgs = (unsigned)F.ks_group, vgs = (unsigned)F.vs_group;
    const unsigned koff = there ? (tok & 31) * kts + f0 / 2 : NOWHERE, ksoff = there ? f0 / CS_FP4_GROUP * kgs + (tok & 31) : NOWHERE;
    const unsigned voff = there ? (tok & 31) * vts + f0 / 2 : NOWHERE, vsoff = there ? f0 / CS_FP4_GROUP * vgs + (tok & 31) : NOWHERE;
    const uint8_t *Kh = F.k + kvh * F.k_head, *Vh = F.v + kvh * F.v_head, *KSh = F.ks + kvh * F.ks_head, *VSh = F.vs + kvh * F.vs_head;
    const int32_t* tab = D.p.table + T.b * D.p.table_stride;

    // A lane has one of the next 64 blocks of 32 tokens: where in the pools it starts, so that a request costs the scalar
    // unit no multiplications.  A block whose page does not exist is read from page 0 and laid down with scale byte 0, as are
    // tokens behind the last one or before every window, whose scales may be anything: their codes are finite then.
    uint64_t at_k = 0, at_v = 0, at_ks = 0, at_vs = 0;
    unsigned long long okay = 0, old = 0;                      // blocks that exist, of these and of the 64 before
    auto pages = [&](int blk0) {
        const int64_t t = (int64_t)w_begin + 32 * ((int64_t)blk0 + lane);
        const int page = t < t_end ? tab[t >> D.page_log2] : -1, slot = (int)t & (D.p.page_size - 32);
        const bool ok = (unsigned)page < (unsigned)D.p.n_pages;
        const int64_t pg = ok ? page : 0;
        old = okay;
        okay = __ballot(ok);
        at_k = (uint64_t)(Kh + pg * F.k_page + slot * F.k_token);
        at_v = (uint64_t)(Vh + pg * F.v_page + slot * F.v_token);
        at_ks = (uint64_t)(KSh + pg * F.ks_page + slot);
        at_vs = (uint64_t)(VSh + pg * F.vs_page + slot);
    };
    unsigned kc[DW], vc[DW], ksc, vsc;
    auto request = [&](int i) {
        if ((2 * i & 63) == 0) pages(2 * i);
        const int l = (2 * i + (wave >> 2)) & 63;
        auto from = [&](uint64_t a) {
            return cs_rsrc((const void*)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(a >> 32), l) << 32 |
                                         (unsigned)__builtin_amdgcn_readlane((int)a, l)), NOWHERE);
        };
        const auto rk = from(at_k), rv = from(at_v), rks = from(at_ks), rvs = from(at_vs);
        const int t = w_begin + 64 * i + tok;
        const bool mine = t < n_lim && t >= w_first && (okay >> l & 1);
        if constexpr (DW == 1) {
            kc[0] = __builtin_amdgcn_raw_buffer_load_b32(rk, koff, 0, 0);
            vc[0] = __builtin_amdgcn_raw_buffer_load_b32(rv, voff, 0, 0);
        } else if constexpr (DW == 2) {
            const auto x = __builtin_amdgcn_raw_buffer_load_b64(rk, koff, 0, 0), y = __builtin_amdgcn_raw_buffer_load_b64(rv, voff, 0, 0);
#pragma unroll
            for (int d = 0; d < DW; ++d) kc[d] = x[d], vc[d] = y[d];
        } else {
            const auto x = __builtin_amdgcn_raw_buffer_load_b128(rk, koff, 0, 0), y = __builtin_amdgcn_raw_buffer_load_b128(rv, voff, 0, 0);
#pragma unroll
            for (int d = 0; d < DW; ++d) kc[d] = x[d], vc[d] = y[d];
        }
        ksc = __builtin_amdgcn_raw_buffer_load_b8(rks, mine ? ksoff : NOWHERE, 0, 0);
        vsc = __builtin_amdgcn_raw_buffer_load_b8(rvs, mine ? vsoff : NOWHERE, 0, 0);
    };
    // where they go: block (wave / 4), half, token of the half
    unsigned char* const put = &stage[0][0] + (wave >> 2) * HALF + (wave >> 1 & 1) * KS * 1024;
    const int row = tok & 15;
    auto lay_down = [&](int buf) {
        unsigned char* p = put + buf * STAGE_BYTES;
#pragma unroll
        for (int d = 0; d < DW; ++d) {
            const int f = f0 + 8 * d;
            *reinterpret_cast<bf16x8*>(p + (f >> 5) * 1024 + (row + 16 * (f >> 3 & 3)) * 16) = cs_fp4_decode(kc[d], ksc << 23);
            *reinterpret_cast<bf16x8*>(p + V_AT + (f >> 5) * 1024 + (f >> 4 & 1) * 512 + row * 32 + (f >> 3 & 1) * 16) = cs_fp4_decode(vc[d], vsc << 23);
        }
    };

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

    auto scores = [&](const unsigned char* sp, f32x4 (&sacc)[2 * NB][NT]) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const f32x4 zero4 = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int a = 0; a < 2 * NB; ++a) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8*>(sp + (a >> 1) * HALF + (((a & 1) * KS + s) * 64 + lane) * 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        sacc[a][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qreg[nt][s][p], s + p == 0 ? zero4 : sacc[a][nt], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // the running maximum of the tile rows moves (and O is rescaled) only when it is left behind by 2^8
    auto reference = [&](const f32x4 (&sacc)[2 * NB][NT], bool masked) {
        if (!masked) {
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float lm = -INFINITY;
#pragma unroll
                for (int a = 0; a < 2 * NB; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) lm = fmaxf(lm, sacc[a][nt][j]);
                over |= !(lm <= thr[nt]);
            }
            if (!__any(over)) return;
        }
        bool moved = false;
        float alpha[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = -INFINITY;
#pragma unroll
            for (int a = 0; a < 2 * NB; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sacc[a][nt][j]);
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
    auto finish = [&](f32x4 (&sacc)[2 * NB][NT], const unsigned char* sp, int t0, auto masked_tag, int ok) {
        constexpr bool masked = decltype(masked_tag)::value;
        if constexpr (masked) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int a = 0; a < 2 * NB; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = t0 + 16 * a + 4 * g + j;
                        const bool sees = t <= q_last[nt] && (A.window == 0 || t > q_last[nt] - A.window) && t < n_lim && (ok >> (a >> 1) & 1);
                        sacc[a][nt][j] = sees ? sacc[a][nt][j] : -INFINITY;
                    }
        }
        reference(sacc, masked);
        bf16x8 pb[NB][NT][NP];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m_safe = m_run[nt] == -INFINITY ? 0.f : m_run[nt];
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(sacc[2 * b + (e >> 2)][nt][e & 3], scale2, -m_safe));
                f4_split8(x, pb[b][nt]);
            }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                s16x4 h[2];
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const unsigned char* p = sp + V_AT + b * HALF + (a * KS + (mt >> 1)) * 1024 + (mt & 1) * 512 + lane * 8;
                    h[a] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) unsigned char*)p);
                }
                const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8){h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]});
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int p = 0; p < NP; ++p) oacc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[b][nt][p], oacc[mt][nt], 0, 0, 0);
            }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int p = 0; p < NP; ++p) lacc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[b][nt][p], lacc[nt], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
    };

    // The loop's bound and the positions come from a vector register that the compiler cannot see through: around branches
    // it takes for uniform it splits the live ranges of the accumulators, copies and spills them.
    int vzero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(vzero));
    const int n_stages_v = n_stages + vzero;
    // positions that this wave's rows have: blocks outside what they see are not computed, blocks inside need no mask
    const int p_lo = T.L + (T.n0 + wave * WROWS) / G + vzero, p_hi = T.L + min(T.rows - 1, (T.n0 + wave * WROWS + WROWS - 1) / G) + vzero;
    const int w_lo = A.window ? p_lo - A.window + 1 : 0, w_hi = A.window ? p_hi - A.window + 1 : 0;
    const int p_end = T.n0 + wave * WROWS < T.QR ? min(p_hi, t_end - 1) : -1;       // a wave without rows multiplies nothing
    const int p_open = min(p_lo, D.cap - 1);
    f32x4 sa[2 * NB][NT];
    if (n_stages > 0) {
        request(0);
        lay_down(0);
        request(1);
    }
    __syncthreads();
    const std::integral_constant<bool, false> plain_tag;
    const std::integral_constant<bool, true> masked_tag;
    for (int i = 0; i < n_stages_v; ++i) {
        const unsigned long long there_are = (i + 1) >> 5 == i >> 5 ? okay : old;
        const int exist = (int)(there_are >> ((2 * i) & 63)) & 3;
#pragma unroll
        for (int b = 0; b < 2; b += NB) {
            const int t0 = w_begin + 64 * i + 32 * b, ok = NB == 2 ? exist : exist >> b & 1;
            const int gone = ((2 * NB - 1) & ~ok) + vzero;
            const unsigned char* sp = stage[i & 1] + b * HALF;
            if (b + NB == 2) {                                  // (past the last stage: what the last request has left, into a half that nobody reads)
                lay_down((i + 1) & 1);
                request(i + 2);
            }
            if ((t0 <= p_end) & (t0 + 32 * NB - 1 >= w_lo)) {
                scores(sp, sa);
                if ((t0 + 32 * NB - 1 > p_open) | (t0 < w_hi) | (gone != 0)) finish(sa, sp, t0, masked_tag, ok);
                else finish(sa, sp, t0, plain_tag, ok);
            }
        }
        __syncthreads();
    }

    // oacc[mt][nt][j]: query row nt*16 + c, feature mt*16 + 4g + j
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = n0 + nt * 16;
        if (n >= T.QR) continue;
        const int i = n / G, h = kvh * G + n - i * G;
        const int64_t r = T.row0 + i, row = ((int64_t)K.entry * KVH + kvh) * P.TR + n - T.n0;
        const float l = lacc[nt][0], inv = l > 0.f ? 1.0f / l : 0.f;
        const bool whole = K.nsplit == 1;
        if (g == 0 && !whole) P.pml[row] = make_float2(m_run[nt], l);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int d = mt * 16 + 4 * g;
            if (d >= hd) continue;
            if (whole) pa_store4((T_*)A.out + r * A.out_row + h * A.out_head + d, oacc[mt][nt] * inv);
            else pa_store4(P.po + row * hd + d, oacc[mt][nt]);
        }
    }
}

// ---- entry points --------------------------------------------------------------------------
static int check_shape(const char* who, const cs_pages_fp4* p, int32_t q_dtype, int32_t n_heads, int32_t R, int32_t max_rows, int64_t max_len) {
    CS_TRY(cs_fp4_check(who, p));
    CS_REQUIRE(q_dtype == CS_F32 || q_dtype == CS_BF16, CS_E_ARG, "%s: queries of unknown type %d", who, q_dtype);
    CS_REQUIRE(n_heads >= 1 && n_heads <= 4096 && n_heads % p->n_kv_heads == 0, CS_E_ARG,
               "%s: n_heads must be a multiple of n_kv_heads, up to 4096", who);
    CS_REQUIRE(R >= 0 && R <= 1 << 26, CS_E_ARG, "%s: R out of range", who);
    CS_REQUIRE((int64_t)R * n_heads <= 1 << 30, CS_E_UNSUPPORTED, "%s: R * n_heads exceeds 2^30", who);
    CS_REQUIRE(max_rows >= 0 && max_len >= 0, CS_E_ARG, "%s: negative max_rows or max_len", who);
    return CS_OK;
}

// Workgroups of the kernel of few rows that run at once: two a compute unit.  (Of 64 features and up to 32 rows three fit; they are
// priced as two.)
#define F4_SLOTS 512
#define F4_LEAST 8                // blocks below which a part of a tile costs more than it saves
// How a call is cut: the same for the workspace and the launches.
struct f4_cut {
    int hdt;
    struct {
        int nt, TR, qr_lo, qr_hi, tiles;      // tiles: an upper bound; 0: no launch
        int W, most, groups;                  // see f4_shares; workgroups per KV head
        float bound, join;
    } narrow;
    pa_part wide;
    int64_t at_w, bytes;                      // where the second launch's partial results start; bytes in all
};
// Workgroups per KV head where all tokens are shared out: two for each compute unit in all, or as many rounds of them as
// leave less than a tenth of the last one idle.
static int f4_share_workgroups(int KVH) {
    for (int slots = F4_SLOTS; slots < 8 * F4_SLOTS; slots *= 2)
        if (slots / KVH * KVH * 10 >= slots * 9) return slots / KVH;
    return std::max(1, 8 * F4_SLOTS / KVH);
}
#define F4N_MOST 48               // query rows up to which a stream takes the kernel of few rows
// KV heads whose rows of codes lie in one cache line of 128 bytes
static int f4_near(const cs_pages_fp4* p) {
    int n = 1;
    while (p->n_kv_heads % (2 * n) == 0 && 2 * n * p->k_head <= 128) n *= 2;
    return n;
}
static f4_cut f4_make_cut(const cs_pages_fp4* p, bool f32, int H, bool has_row0, int R, int max_rows, int64_t max_len) {
    f4_cut c = {};
    const int KVH = p->n_kv_heads, G = H / KVH, B = p->batch, cap = p->table_pages * p->page_size;
    const int rows = has_row0 ? (max_rows ? std::min(max_rows, R) : R) : R / B;
    const int64_t qr = (int64_t)rows * G, all = (int64_t)R * G, len = max_len && max_len < cap ? max_len : cap;
    c.hdt = p->head_dim <= 64 ? 64 : p->head_dim <= 128 ? 128 : 256;
    auto& N = c.narrow;
    pa_part& W = c.wide;
    // Streams of up to n_most query rows per KV head go to the kernel of few rows.  Where a batch has
    // longer ones too, that kernel is made for single tokens: a tile of 48 rows would cost every one of
    // them three tiles' products.
    const int n_most = c.hdt == 256 || qr > F4N_MOST ? 16 : F4N_MOST;
    if (has_row0 || qr <= n_most) {
        N.nt = (int)std::min<int64_t>(n_most / 16, cs_ceil_div(qr, 16));
        N.TR = 16 * N.nt;
        N.qr_hi = qr <= n_most ? 0x7fffffff : n_most;
        N.tiles = !has_row0 ? B : (int)(qr <= n_most ? all / N.TR + std::min(B, R) : std::min(B, R));
    }
    if (qr > n_most) {
        // Tiles of half the rows where whole ones, cut into ranges of 256 tokens of what a row sees on
        // average, leave the chip unfilled.  (The price of a cut seldom goes as fine: 1581 rows of 16 heads on an empty cache are 112
        // whole tiles, their ranges and a merge, 49 us for 8 us of multiplies.)
        const bool unfilled = (all / (F4W_WAVES * 32) + 1) * KVH * std::max<int64_t>(1, (len - rows / 2) / 256) < 256;
        auto tiles = [&](int TR) { return has_row0 ? all / TR + std::min<int64_t>(B, all / (n_most + 1)) : B * cs_ceil_div(qr, TR); };
        // Of 64 features and half the rows two workgroups run on a compute unit at once, and whole tiles that fill the chip come out
        // more even: 2500 rows of 28 heads, 4 KV heads 74 -> 50 us, behind 4000 195 -> 173, 8 x 700 behind 1000 113 -> 102, behind
        // 16000 1024 -> 883.  Up to twice as many as compute units are cut over a long context, into more partial results
        // then (2500 rows of 28 heads behind 16000 484 -> 561), as are fewer (8 x 700 rows of 4 heads behind 4000 67 -> 80).
        const int64_t items = tiles(F4W_WAVES * 32) * KVH;
        const bool even = c.hdt == 64 && items >= (len <= 8192 ? 256 : 512);
        W.nt = c.hdt == 256 || f32 || unfilled || even ? 1 : 2;
        W.TR = F4W_WAVES * 16 * W.nt;
        W.qr_lo = has_row0 ? n_most : 0;
        W.qr_hi = 0x7fffffff;
        W.tiles = (int)tiles(W.TR);
    }
    if (N.tiles) {
        // What a block of 32 tokens takes a workgroup that runs alone (captured calls: 4.3, 5.2 and 6.6 ns a token of 64, 128
        // and 256 features, 16 bfloat16 rows; 8.6 with 48 rows, 8.3 and 19.2 with 16 and 48 float32 rows), and what it costs the
        // chip: its bytes at 5 TB/s, or one of the 256 compute units for as long.
        const float alone = 0.032f * (3.6f + 0.0125f * c.hdt) * (0.7f + 0.32f * N.nt * (f32 ? 3 : 1));
        const float chip = std::max(0.00087f * p->head_dim / 128, alone / 256);
        N.bound = KVH * chip / alone;
        N.join = 5.0f / alone;                                   // (a merge: 5 us; one that finds nothing to do: 3)
        const int share = f4_share_workgroups(KVH), tiles = N.tiles;
        auto price = [&](float longest, float all) { return std::cbrt(longest * longest * longest + all * all * all); };
        const float blocks = cs_ceil_div(len, 32), chip_all = blocks * tiles * N.bound, whole = price(blocks, chip_all);
        const float cut = price(std::max(blocks * tiles / share, (float)F4_LEAST), chip_all) + N.join;
        // (Tables of 2^24 tokens and 960 tiles; wider ones with more tiles leave each one whole.  A bound that let every stream have all
        // rows left 15 single tokens beside 8192 rows uncut from 2^19 on, 32 heads over 2 KV heads: 2350 -> 2413 us.)
        const int64_t most = (int64_t)tiles * (cap / 32 + 1 + F4_SEGMENT);
        const bool fits = most < 1 << 29;
        // Streams of one length gain by that; others may where the longest alone takes ten times what a merge costs.  Twice as
        // many tiles as workgroups even out by themselves.
        if (fits && tiles < 2 * share && (cut < whole || (tiles > 1 && blocks > 10 * N.join))) N.W = share, N.most = (int)most;
        // (without shares: as f4_start counts them)
        N.groups = N.W ? N.W : !has_row0 || N.qr_hi <= N.TR ? (has_row0 ? B : tiles) : (int)(all / N.TR) + B;
    }
    c.at_w = N.W ? cs_round_up((int64_t)2 * N.W * KVH * N.TR * (p->head_dim * 4 + 8), 16) + (int64_t)2 * N.W * 16 : 0;
    // A workgroup's ends and the merge in tokens of the kernel for many rows (with 128 and 192 for bfloat16 queries too: 4 x
    // 300 rows of 32 heads behind 1000 tokens 52 -> 70 us, behind 16000 344 -> 399, 33 rows of 16 heads of 64 behind 300
    // 14 -> 15; with 256 and 400 for float32 ones 33 rows of 8 heads behind 300 24 -> 26, 100 rows 25 -> 29).  256 workgroups
    // run at once, one a compute unit; the two of 64 features and half the rows count as one.
    c.bytes = c.at_w + (f32 ? pa_ranges(W, len, B, KVH, p->head_dim, 256, 128, 192) : pa_ranges(W, len, B, KVH, p->head_dim, 256, 256, 400));
    return c;
}

extern "C" int64_t cs_paged_fp4_attention_workspace(const cs_pages_fp4* p, int32_t q_dtype, int32_t n_heads, int32_t has_row0, int32_t R,
                                                    int32_t max_rows, int64_t max_len) {
    const char* who = "cs_paged_fp4_attention_workspace";
    CS_TRY(check_shape(who, p, q_dtype, n_heads, R, max_rows, max_len));
    CS_REQUIRE(has_row0 || p->batch == 0 || R % p->batch == 0, CS_E_ARG, "%s: R rows cannot be shared out among %d streams without d_row0",
               who, p->batch);
    if (R == 0 || p->batch == 0) return 0;
    return f4_make_cut(p, q_dtype == CS_F32, n_heads, has_row0 != 0, R, max_rows, max_len).bytes;
}

template <int HD, int NT, int NP, bool KLDS = false>
static int f4n_launch(const cs_fp4_dev& F, const pa_args& A, const f4_shares& S, dim3 grid, hipStream_t s) {
    k_paged_fp4_narrow<HD, NT, NP, KLDS><<<grid, 64 * F4N_WAVES, 0, s>>>(f4_call{F, A, S});
    return cs_launch_ok("k_paged_fp4_narrow");
}
template <int HD, int NT, int NP>
static int f4w_launch(const cs_fp4_dev& F, const pa_args& A, const pa_plan& P, dim3 grid, hipStream_t s) {
    k_paged_fp4_wide<HD, NT, NP><<<grid, 64 * F4W_WAVES, 0, s>>>(F, A, P);
    return cs_launch_ok("k_paged_fp4_wide");
}

extern "C" int cs_paged_fp4_attention(const cs_pages_fp4* p, int32_t q_dtype, const void* q, int64_t q_row, int64_t q_head, int32_t n_heads,
                                      const int32_t* d_row0, int32_t R, float scale, int32_t window, int32_t max_rows, int64_t max_len,
                                      void* out, int64_t out_row, int64_t out_head, void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "cs_paged_fp4_attention";
    CS_TRY(check_shape(who, p, q_dtype, n_heads, R, max_rows, max_len));
    CS_REQUIRE(scale > 0.f && std::isfinite(scale), CS_E_ARG, "%s: scale must be positive and finite", who);
    CS_REQUIRE(window >= 0, CS_E_ARG, "%s: negative window", who);
    cs_fp4_dev F;
    CS_TRY(cs_fp4_view(who, p, d_row0, R, &F));
    if (R == 0 || p->batch == 0) return CS_OK;
    const bool f32 = q_dtype == CS_F32;
    const size_t esz = f32 ? 4 : 2;
    CS_TRY(cs_check_rows(who, "q", q, q_row, q_head, esz));
    CS_TRY(cs_check_rows(who, "out", out, out_row, out_head, esz));
    CS_TRY(cs_check_apart(who, "out", out_row, R, out_head, n_heads, p->head_dim));
    F.d.p.dtype = q_dtype;                                      // (the merge's outputs)
    const pa_args A = {q, q_row, q_head, out, out_row, out_head, n_heads, n_heads / p->n_kv_heads, window, scale * 1.4426950408889634f};
    hipStream_t s = (hipStream_t)stream;
    const f4_cut c = f4_make_cut(p, f32, n_heads, d_row0 != nullptr, R, max_rows, max_len);
    CS_REQUIRE(c.bytes <= 0 || (workspace && workspace_bytes >= c.bytes), CS_E_CAPACITY, "%s: the workspace has %lld bytes, %lld are needed",
               who, (long long)(workspace ? workspace_bytes : 0), (long long)c.bytes);
    CS_REQUIRE(((uintptr_t)workspace & 15) == 0, CS_E_ARG, "%s: the workspace is not aligned to 16 bytes", who);
    const int64_t grid_n = (int64_t)c.narrow.groups * p->n_kv_heads, grid_w = (int64_t)c.wide.entries * p->n_kv_heads;
    CS_REQUIRE(grid_n <= 0x7fffffff && grid_w <= 0x7fffffff, CS_E_UNSUPPORTED, "%s: too many tiles", who);
    int rc = CS_E_UNSUPPORTED;
    if (grid_w) {
        const pa_plan P = pa_plan_of(c.wide, (char*)workspace + c.at_w, p->n_kv_heads, p->head_dim);
        const dim3 n = cs_paged_grid(grid_w);
#define FW(HD_, NT_) if (c.hdt == HD_ && c.wide.nt == NT_) rc = NT_ == 1 && f32 ? f4w_launch<HD_, 1, 3>(F, A, P, n, s) : f4w_launch<HD_, NT_, 1>(F, A, P, n, s)
        FW(64, 1); FW(64, 2); FW(128, 1); FW(128, 2); FW(256, 1);
#undef FW
        CS_TRY(rc);
        // (a merge waits for its loads: up to eight workgroups for one, where the chip has room for them: 700 and 438 float32 rows behind
        // 3001 and 1876 83 -> 76 us, with two 79; 6 x 3269 rows of 4 heads 166 -> 163; 16 x 33 of 28 heads behind 65535 502 -> 497)
        CS_TRY(pm_launch(F.d, A, P, dim3(n.x, (unsigned)std::clamp<int64_t>(4096 / grid_w, 1, 8), n.z), s));
    }
    if (grid_n) {
        const auto& N = c.narrow;
        const int64_t rows = (int64_t)2 * N.W * p->n_kv_heads * N.TR;
        float* po = (float*)workspace;
        const f4_shares S = {N.TR, N.qr_lo, N.qr_hi, N.W, F4_LEAST, N.W ? (N.W + 63) / 64 : N.groups, N.bound, N.join, f4_near(p), N.most, po, (float2*)(po + rows * p->head_dim),
                             (int4*)((char*)workspace + cs_round_up(rows * (p->head_dim * 4 + 8), 16))};
        const dim3 n = cs_paged_grid(grid_n);
#define FN(HD_, NT_) if (c.hdt == HD_ && N.nt == NT_) rc = f32 ? f4n_launch<HD_, NT_, 3>(F, A, S, n, s) : f4n_launch<HD_, NT_, 1>(F, A, S, n, s)
        if (c.hdt == 128 && N.nt == 1 && !f32 && p->k_token > p->head_dim / 2) rc = f4n_launch<128, 1, 1, true>(F, A, S, n, s);
        else FN(128, 1);
        FN(64, 1); FN(64, 2); FN(64, 3); FN(128, 2); FN(128, 3); FN(256, 1);
#undef FN
        CS_TRY(rc);
        if (N.W) {
            int lanes = 0;
            while (4 << lanes < p->head_dim) ++lanes;
            if (f32) k_paged_fp4_join<float><<<n, F4J_THREADS, 0, s>>>(F.d, A, S, lanes);
            else k_paged_fp4_join<bf16_t><<<n, F4J_THREADS, 0, s>>>(F.d, A, S, lanes);
            CS_TRY(cs_launch_ok("k_paged_fp4_join"));
        }
    }
    return CS_OK;
}
