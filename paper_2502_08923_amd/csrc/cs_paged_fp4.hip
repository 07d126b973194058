// What goes into a paged cache of 4-bit elements and what comes out of it again: the append quantises new
// key and value rows into the pages of their streams (Sec. 3.2: the block is appended to the context; App.
// B.1-B.2: the per-layer K, V), the read gives the values back.
//
//   s = 2^e, the smallest with max|x| <= 7 s over a group of 32;   code = e2m1(x / s);   value = e2m1(code) s
//
// Both are streams of memory: a lane has eight consecutive elements of a head's row (16 bytes of a
// bfloat16 row, one dword of codes), four neighbours have a group.  With x = 2^e' m, 1 <= m < 2, the scale's
// exponent is e' - 2, one more where m > 7/4: an addition to the bits of max|x| that carries into the exponent
// there, so scale and codes are exact integer and power-of-two arithmetic and one rounding.  A thread keeps its head
// and segment and goes from row to row; the places of up to 64 rows are looked up by a wave at once, a lane a row, and
// go round through LDS.  (With a division and three 64-bit products per (row, head) pair instead, the vector unit was
// the bound: append of 11 thousand rows of 8 heads of 128 16.9 us -> 12.8, read of 145 thousand 282 -> 204, 123 with
// stores past the caches, 108 with neighbours on one die: 4.2 and 7.0 TB/s.)  88 rows take 3.6 us either way, a launch's latency.
#include <algorithm>

#include "cs_paged_fp4.h"

// ---- argument checks -------------------------------------------------------------------
#define CS_MAX_BSTRIDE ((int64_t)1 << 40)

static int check_pool(const char* who, const char* name, const void* base, int64_t page, int64_t head, int64_t inner, int64_t least,
                      int64_t steps, int64_t width) {
    CS_TRY(cs_check_rows(who, name, base, page, head, 1));
    CS_REQUIRE(steps < 2 || inner >= least, CS_E_ARG, "%s: an inner stride of %s is less than %lld bytes", who, name, (long long)least);
    CS_REQUIRE(inner >= 0 && inner <= CS_MAX_BSTRIDE && inner % 16 == 0, CS_E_ARG, "%s: an inner stride of %s is no multiple of 16 bytes", who, name);
    CS_REQUIRE((steps - 1) * inner + width < (int64_t)1 << 31, CS_E_UNSUPPORTED, "%s: a page of %s spans 2^31 bytes or more", who, name);
    return CS_OK;
}

int cs_fp4_check(const char* who, const cs_pages_fp4* p) {
    CS_REQUIRE(p, CS_E_ARG, "%s: NULL pages", who);
    CS_REQUIRE(p->reserved[0] == 0 && p->reserved[1] == 0, CS_E_ARG, "%s: a reserved field is not 0", who);
    CS_REQUIRE(p->batch >= 0 && p->n_pages >= 1 && p->n_kv_heads >= 1 && p->table_pages >= 1, CS_E_ARG,
               "%s: a size of the pages is out of range", who);
    CS_REQUIRE(p->batch == 0 || (p->table && p->len), CS_E_ARG, "%s: NULL table or lengths", who);
    CS_REQUIRE(p->table_stride >= p->table_pages, CS_E_ARG, "%s: table_stride is less than table_pages", who);
    CS_REQUIRE(p->head_dim >= 32 && p->head_dim <= 256 && p->head_dim % 32 == 0, CS_E_UNSUPPORTED,
               "%s: head_dim must be a multiple of 32 in 32..256", who);
    CS_REQUIRE(p->page_size >= 32 && p->page_size <= 32768 && (p->page_size & (p->page_size - 1)) == 0, CS_E_UNSUPPORTED,
               "%s: page_size must be a power of two in 32..32768", who);
    CS_REQUIRE((int64_t)p->table_pages * p->page_size <= (int64_t)1 << 30, CS_E_UNSUPPORTED,
               "%s: table_pages * page_size exceeds 2^30", who);
    CS_REQUIRE(p->batch <= 65536 && p->n_kv_heads <= 4096, CS_E_UNSUPPORTED, "%s: too many streams or heads", who);
    const int hd = p->head_dim, P = p->page_size;
    CS_TRY(check_pool(who, "k", p->k, p->k_page, p->k_head, p->k_token, hd / 2, P, hd / 2));
    CS_TRY(check_pool(who, "v", p->v, p->v_page, p->v_head, p->v_token, hd / 2, P, hd / 2));
    CS_TRY(check_pool(who, "k_scale", p->k_scale, p->ks_page, p->ks_head, p->ks_group, P, hd / CS_FP4_GROUP, P));
    CS_TRY(check_pool(who, "v_scale", p->v_scale, p->vs_page, p->vs_head, p->vs_group, P, hd / CS_FP4_GROUP, P));
    return CS_OK;
}

int cs_fp4_view(const char* who, const cs_pages_fp4* p, const int32_t* d_row0, int32_t R, cs_fp4_dev* d) {
    cs_pages q = {};
    q.table = p->table, q.table_stride = p->table_stride, q.len = p->len;
    q.batch = p->batch, q.table_pages = p->table_pages, q.n_pages = p->n_pages, q.page_size = p->page_size;
    q.n_kv_heads = p->n_kv_heads, q.head_dim = p->head_dim, q.dtype = CS_BF16;
    CS_TRY(cs_pages_view(who, &q, d_row0, R, &d->d));
    d->k = p->k, d->v = p->v, d->ks = p->k_scale, d->vs = p->v_scale;
    d->k_page = p->k_page, d->k_head = p->k_head, d->k_token = p->k_token;
    d->v_page = p->v_page, d->v_head = p->v_head, d->v_token = p->v_token;
    d->ks_page = p->ks_page, d->ks_head = p->ks_head, d->ks_group = p->ks_group;
    d->vs_page = p->vs_page, d->vs_head = p->vs_head, d->vs_group = p->vs_group;
    return CS_OK;
}

// ---- rows and their places --------------------------------------------------------------
#define F4_THREADS 256
#define F4_ROWS 64            // most rows of a workgroup: a lane each for their places
// Rows of a thread in flight, and in all.  (Captured calls.  Append with two, four and eight in flight: 160 thousand rows of one head of
// 64 12.7, 14.9 and 16.3 us, 11 thousand of 8 heads of 128 13.1, 13.8 and 18.1; read with two, four and eight: 145 thousand rows of 8
// heads 108.5, 107.9 and 108.5, 11 thousand 12.5, 12.4 and 12.6.  Four, eight and 16 rows of a thread, for both: the same append 14.6,
// 13.4 and 13.8, the same reads 103, 108 and 112, and 11.2, 12.4 and 12.6.)
#define F4_APPEND_BATCH 2
#define F4_READ_BATCH 4
#define F4_PASSES 8

struct f4_side {
    void* rows;
    int64_t row, head;
};
struct f4_args {
    f4_side s[2];             // keys, values
    const int32_t* first;     // position of row 0 of every stream, or NULL: its length
    int rpw, lanes_log2, segs;
};

// (page, position) of row r0 + lane, for the nr lanes of a wave that have one; page -1: nowhere, -2: nobody's row
// (first: position of every stream's row 0, or NULL: its length)
__device__ __forceinline__ int2 f4_place(const cs_pages_dev& D, const int32_t* first, int r0, int nr, int lane) {
    const int B = D.p.batch, r = r0 + lane;
    int b = B;
    if (!D.row0) b = r / D.rows;
    else if (B <= 64) {
        // as many streams end at or before a row: one load, and a count over the wave for every row
        const int end = lane < B ? D.row0[lane + 1] : 0x7fffffff;
        for (int i = 0; i < nr; ++i) {
            const int n = __popcll(__ballot(end <= r0 + i));
            b = lane == i ? n : b;
        }
    } else {
        int lo = 0, hi = B;                                      // the first stream that ends behind the row
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const bool ended = D.row0[mid + 1] <= r;
            lo = ended ? mid + 1 : lo;
            hi = ended ? hi : mid;
        }
        b = lo;
    }
    if (lane >= nr || b >= B) return make_int2(-2, 0);
    const int2 sr = cs_stream_rows(D, b);
    if (r < sr.x || r - sr.x >= sr.y) return make_int2(-2, 0);
    const int64_t at = (int64_t)(first ? first[b] : cs_stream_len(D, b)) + (r - sr.x);
    if (at < 0 || at >= D.cap) return make_int2(-1, 0);
    const int page = D.p.table[b * D.p.table_stride + (at >> D.page_log2)];
    return make_int2(page < 0 || page >= D.p.n_pages ? -1 : page, (int)at);
}

// What a thread has: one segment of one head (keys' heads before values') in every `step`-th row of the workgroup's,
// from row `r` on, so that all addresses but the place of a row are made once.  Heads that the threads do not reach
// at once come in further rounds.
struct f4_mine {
    bool on, is_v;
    int r, step, g, seg;
    __device__ __forceinline__ f4_mine(const f4_args& A, int KVH, int tid, int round) {
        const int lanes = 1 << A.lanes_log2, heads = 2 * KVH, teams = F4_THREADS >> A.lanes_log2;
        seg = tid & (lanes - 1);
        step = max(teams / heads, 1);
        const int team = tid >> A.lanes_log2, q = heads < teams ? team % heads : team, h = round * teams + q;
        r = heads < teams ? team / heads : 0;
        on = seg < A.segs && h < heads && r < step;
        is_v = h >= KVH;
        g = is_v ? h - KVH : h;
    }
};
// where a row's codes and scales of head 0 lie in their pools, keys and values; of codes -1: nowhere, -2: nobody's row
struct f4_places {
    longlong2 at[2][F4_ROWS];
    __device__ __forceinline__ void set(const cs_fp4_dev& F, int i, int2 p) {
        const int64_t slot = p.y & (F.d.p.page_size - 1);
        const bool some = p.x >= 0;
        at[0][i] = make_longlong2(some ? p.x * F.k_page + slot * F.k_token : p.x, p.x * F.ks_page + slot);
        at[1][i] = make_longlong2(some ? p.x * F.v_page + slot * F.v_token : p.x, p.x * F.vs_page + slot);
    }
};

template <typename T>
struct f4_raw;
template <>
struct f4_raw<bf16_t> { u32x4 x; };
template <>
struct f4_raw<float> { f32x4 x[2]; };
__device__ __forceinline__ void f4_load(f4_raw<bf16_t>& o, const bf16_t* p) { o.x = *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void f4_load(f4_raw<float>& o, const float* p) {
    o.x[0] = *reinterpret_cast<const f32x4*>(p);
    o.x[1] = *reinterpret_cast<const f32x4*>(p + 4);
}
__device__ __forceinline__ void f4_floats(const f4_raw<bf16_t>& r, float* o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        o[2 * j] = __uint_as_float(r.x[j] << 16);
        o[2 * j + 1] = __uint_as_float(r.x[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void f4_floats(const f4_raw<float>& r, float* o) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = r.x[j >> 2][j & 3];
}

// the largest of the four lanes of a quad
__device__ __forceinline__ unsigned f4_quad_max(unsigned v) {
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));       // lanes 1 0 3 2
    return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
}

// The workgroup's turn.  Dies take workgroups in turn, eight of them, each with a cache of its own: RUN neighbours, whose
// rows share lines of scales, are eight workgroups apart.  (Read of 145 thousand rows of 8 heads, pages of 64: runs of 1 124 us, 8
// 112, 64 108, 256 110; append of 11 thousand 14.1, 13.5, 13.8, 14.1, of 4096 7.8, 7.6, 7.4, 7.8.)
#define F4_APPEND_RUN 8
#define F4_READ_RUN 64
template <int RUN>
__device__ __forceinline__ int f4_turn() {
    const int n = gridDim.x * gridDim.z, wg = (int)cs_paged_wg(), i = wg & (8 * RUN - 1);
    return (wg | (8 * RUN - 1)) < n ? wg - i + (i & 7) * RUN + (i >> 3) : wg;
}

// ---- append -----------------------------------------------------------------------------

template <typename TI>
__global__ __launch_bounds__(F4_THREADS) void k_paged_fp4_append(cs_fp4_dev F, f4_args A) {
    __shared__ f4_places to;
    const cs_pages_dev& D = F.d;
    const int tid = threadIdx.x, KVH = D.p.n_kv_heads;
    const int r0 = f4_turn<F4_APPEND_RUN>() * A.rpw, nr = min(A.rpw, D.R - r0);
    // rows behind the last stream are not read; the others are in flight while their places are looked up
    const int live = D.row0 ? min(nr, min(max(D.row0[D.p.batch], 0), D.R) - r0) : nr;
    for (int round = 0; round * (F4_THREADS >> A.lanes_log2) < 2 * KVH; ++round) {
        const f4_mine M(A, KVH, tid, round);
        const f4_side& side = A.s[M.is_v];
        const TI* src = (const TI*)side.rows + (int64_t)(r0 + M.r) * side.row + (int64_t)M.g * side.head + M.seg * 8;
        const int64_t src_step = M.step * side.row;
        uint8_t* codes_at = (M.is_v ? F.v + M.g * F.v_head : F.k + M.g * F.k_head) + M.seg * 4;
        uint8_t* scales_at = M.is_v ? F.vs + M.g * F.vs_head + (M.seg >> 2) * F.vs_group : F.ks + M.g * F.ks_head + (M.seg >> 2) * F.ks_group;
        f4_raw<TI> x[F4_APPEND_BATCH];
        int r = M.on ? M.r : live;
        auto request = [&](int r) {
#pragma unroll
            for (int u = 0; u < F4_APPEND_BATCH; ++u) {
                if (r + u * M.step < live) f4_load(x[u], src);
                src += src_step;
            }
        };
        request(r);
        if (round == 0) {
            if (tid < CS_WAVE) {
                const int2 at = f4_place(D, nullptr, r0, nr, tid);
                if (tid < nr) to.set(F, tid, at);
            }
            __syncthreads();
        }
        for (; r < live; r += F4_APPEND_BATCH * M.step) {
#pragma unroll
            for (int u = 0; u < F4_APPEND_BATCH; ++u) {
                if (r + u * M.step >= live) break;
                float v[8];
                f4_floats(x[u], v);
                unsigned top = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
                top = f4_quad_max(top);                        // (of integers: a NaN counts as more than an infinity)
                const int e = (int)((top + 0x1fffffu) >> 23) - 2;
                const unsigned scale = top >= 0x7f800000u ? 255u : (unsigned)min(max(e, CS_FP4_SCALE_MIN), CS_FP4_SCALE_MAX);
                const float s = __uint_as_float(scale << 23);
                unsigned codes = 0;
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0], v[1], s, 0);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2], v[3], s, 1);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[4], v[5], s, 2);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[6], v[7], s, 3);
                const longlong2 at = to.at[M.is_v][r + u * M.step];
                if (at.x >= 0) {
                    *reinterpret_cast<unsigned*>(codes_at + at.x) = codes;
                    if ((M.seg & 3) == 0) scales_at[at.y] = (uint8_t)scale;
                }
            }
            request(r + F4_APPEND_BATCH * M.step);
        }
    }
}

// ---- read -------------------------------------------------------------------------------
// What a lane has of a row, segment `seg` of `segs` with eight elements each, as numbers.  Stores pass the caches by (12 streams of up
// to 18431 tokens, bfloat16: 165 us through them, 108 past).  A float32 row is twice as long as what one store of its lanes holds: one has
// the first half of the row, one the second, and a lane asks another (`first` and on) for its four codes, for stores that
// leave every other 16 bytes out reach memory in parts (35 thousand rows of 8 heads of 128: 53 us, 153 with such stores, 91 with
// those through the caches).  Halves that are no whole lines go through the caches for the same reason: WHOLE false, heads of 96 41 us for
// 51, of 160 44 for 52, of 64 28 for 29; of 128 and 256 73 for 53.
template <bool WHOLE>
__device__ __forceinline__ void f4_store(bf16_t* row, int seg, int, int, unsigned codes, unsigned scale) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, cs_fp4_decode(codes, scale << 23)), reinterpret_cast<u32x4*>(row + seg * 8));
}
template <bool WHOLE>
__device__ __forceinline__ void f4_store(float* row, int seg, int segs, int first, unsigned codes, unsigned scale) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int q = half * segs + seg, from = first + (q >> 1);
        const bf16x8 v = cs_fp4_decode(__shfl(codes, from, CS_WAVE) >> 16 * (q & 1), __shfl(scale, from, CS_WAVE) << 23);
        const f32x4 o = (f32x4){(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        f32x4* at = reinterpret_cast<f32x4*>(row + q * 4);
        if constexpr (WHOLE) __builtin_nontemporal_store(o, at);
        else *at = o;
    }
}

template <typename TO, bool WHOLE>
__global__ __launch_bounds__(F4_THREADS) void k_paged_fp4_read(cs_fp4_dev F, f4_args A) {
    __shared__ f4_places from;
    const cs_pages_dev& D = F.d;
    const int tid = threadIdx.x, KVH = D.p.n_kv_heads;
    const int r0 = f4_turn<F4_READ_RUN>() * A.rpw, nr = min(A.rpw, D.R - r0);
    const int first_lane = tid & (CS_WAVE - 1) & -(1 << A.lanes_log2);               // of the row's
    if (tid < CS_WAVE) {
        const int2 at = f4_place(D, A.first, r0, nr, tid);
        if (tid < nr) from.set(F, tid, at);
    }
    __syncthreads();
    for (int round = 0; round * (F4_THREADS >> A.lanes_log2) < 2 * KVH; ++round) {
        const f4_mine M(A, KVH, tid, round);
        if (!M.on) continue;
        const f4_side& side = A.s[M.is_v];
        TO* dst = (TO*)side.rows + (int64_t)(r0 + M.r) * side.row + (int64_t)M.g * side.head;
        const int64_t dst_step = M.step * side.row;
        const uint8_t* codes_at = (M.is_v ? F.v + M.g * F.v_head : F.k + M.g * F.k_head) + M.seg * 4;
        const uint8_t* scales_at = M.is_v ? F.vs + M.g * F.vs_head + (M.seg >> 2) * F.vs_group : F.ks + M.g * F.ks_head + (M.seg >> 2) * F.ks_group;
        for (int r = M.r; r < nr; r += F4_READ_BATCH * M.step) {
            unsigned codes[F4_READ_BATCH], scale[F4_READ_BATCH];
            bool mine[F4_READ_BATCH];
#pragma unroll
            for (int u = 0; u < F4_READ_BATCH; ++u) {
                const longlong2 at = from.at[M.is_v][min(r + u * M.step, nr - 1)];
                codes[u] = scale[u] = 0;
                mine[u] = r + u * M.step < nr && at.x != -2;
                if (mine[u] && at.x >= 0) {
                    codes[u] = *reinterpret_cast<const unsigned*>(codes_at + at.x);
                    scale[u] = scales_at[at.y];
                }
            }
#pragma unroll
            for (int u = 0; u < F4_READ_BATCH; ++u) {
                if (mine[u]) f4_store<WHOLE>(dst, M.seg, A.segs, first_lane, codes[u], scale[u]);
                dst += dst_step;
            }
        }
    }
}

// ---- entry points -----------------------------------------------------------------------
// what both have of their arguments; rows per workgroup: see the calls
static int f4_prepare(const char* who, const cs_pages_fp4* p, int32_t dtype, const void* k, int64_t k_row, int64_t k_head, const void* v,
                      int64_t v_row, int64_t v_head, const int32_t* d_row0, int32_t R, cs_fp4_dev* F, f4_args* A) {
    CS_TRY(cs_fp4_check(who, p));
    CS_REQUIRE(dtype == CS_F32 || dtype == CS_BF16, CS_E_ARG, "%s: rows of unknown type %d", who, dtype);
    CS_TRY(cs_fp4_view(who, p, d_row0, R, F));
    if (R == 0 || p->batch == 0) return CS_OK;
    const size_t esz = dtype == CS_BF16 ? 2 : 4;
    CS_TRY(cs_check_rows(who, "k rows", k, k_row, k_head, esz));
    CS_TRY(cs_check_rows(who, "v rows", v, v_row, v_head, esz));
    A->s[0] = {(void*)k, k_row, k_head};
    A->s[1] = {(void*)v, v_row, v_head};
    A->segs = p->head_dim / 8;
    A->lanes_log2 = 2;
    while (1 << A->lanes_log2 < A->segs) ++A->lanes_log2;
    return CS_OK;
}
static int f4_rows_of(const f4_args& A, const cs_pages_fp4* p, int R) {
    // a thread has a segment in some rows, so that the look-up of the places is shared, while there are more than enough
    // rows for the chip
    const int step = std::max(1, (F4_THREADS >> A.lanes_log2) / (2 * p->n_kv_heads));
    return std::max(1, std::min(std::min(F4_PASSES * step, F4_ROWS), R / 1024));
}

extern "C" int cs_paged_fp4_append(const cs_pages_fp4* p, int32_t src_dtype, const void* k, int64_t k_row, int64_t k_head, const void* v,
                                   int64_t v_row, int64_t v_head, const int32_t* d_row0, int32_t R, void* stream) {
    const char* who = "cs_paged_fp4_append";
    cs_fp4_dev F;
    f4_args A = {};
    CS_TRY(f4_prepare(who, p, src_dtype, k, k_row, k_head, v, v_row, v_head, d_row0, R, &F, &A));
    if (R == 0 || p->batch == 0) return CS_OK;
    const int half = p->head_dim / 2, P = p->page_size;
    CS_TRY(cs_check_apart(who, "k", p->k_page, p->n_pages, p->k_head, p->n_kv_heads, half));
    CS_TRY(cs_check_apart(who, "v", p->v_page, p->n_pages, p->v_head, p->n_kv_heads, half));
    CS_TRY(cs_check_apart(who, "k_scale", p->ks_page, p->n_pages, p->ks_head, p->n_kv_heads, P));
    CS_TRY(cs_check_apart(who, "v_scale", p->vs_page, p->n_pages, p->vs_head, p->n_kv_heads, P));
    A.rpw = f4_rows_of(A, p, R);
    const dim3 grid = cs_paged_grid(cs_ceil_div(R, A.rpw));
    hipStream_t s = (hipStream_t)stream;
    if (src_dtype == CS_BF16) k_paged_fp4_append<bf16_t><<<grid, F4_THREADS, 0, s>>>(F, A);
    else k_paged_fp4_append<float><<<grid, F4_THREADS, 0, s>>>(F, A);
    return cs_launch_ok("k_paged_fp4_append");
}

extern "C" int cs_paged_fp4_read(const cs_pages_fp4* p, int32_t dst_dtype, void* k, int64_t k_row, int64_t k_head, void* v, int64_t v_row,
                                 int64_t v_head, const int32_t* d_row0, const int32_t* first, int32_t R, void* stream) {
    const char* who = "cs_paged_fp4_read";
    cs_fp4_dev F;
    f4_args A = {};
    CS_TRY(f4_prepare(who, p, dst_dtype, k, k_row, k_head, v, v_row, v_head, d_row0, R, &F, &A));
    if (R == 0 || p->batch == 0) return CS_OK;
    CS_TRY(cs_check_apart(who, "k rows", k_row, R, k_head, p->n_kv_heads, p->head_dim));
    CS_TRY(cs_check_apart(who, "v rows", v_row, R, v_head, p->n_kv_heads, p->head_dim));
    A.first = first;
    A.rpw = f4_rows_of(A, p, R);
    const dim3 grid = cs_paged_grid(cs_ceil_div(R, A.rpw));
    hipStream_t s = (hipStream_t)stream;
    if (dst_dtype == CS_BF16) k_paged_fp4_read<bf16_t, true><<<grid, F4_THREADS, 0, s>>>(F, A);
    else if (A.segs % 16 == 0) k_paged_fp4_read<float, true><<<grid, F4_THREADS, 0, s>>>(F, A);
    else k_paged_fp4_read<float, false><<<grid, F4_THREADS, 0, s>>>(F, A);
    return cs_launch_ok("k_paged_fp4_read");
}
