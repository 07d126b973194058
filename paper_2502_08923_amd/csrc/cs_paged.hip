// What goes into a paged cache: the norms of query and key heads with the rotary embedding, and the
// append of new key and value rows to the pages of their streams (Sec. 3.2: the block is appended to
// the context; App. B.1-B.2: the per-layer K, V it is appended to).
//
// Both are streams of memory with a little arithmetic on the way.  A workgroup takes a few rows with
// all their heads, so that the angles of a row (head-independent, two float64 products and two series
// each) are made once and shared through LDS, instead of once per head: at 40 heads that is the
// difference between the vector unit and the memory being the bound.  A lane holds VEC consecutive
// elements of a head's first half and the VEC elements of its second half that pair up with them, so
// the rotation needs no other lane; the norm is a shuffle sum over the head's lanes.  Measured: norms
// and rotation of 4096 rows of 40 heads of 128 (84 MB moved) 17.0 to 17.5 us = 4.8 to 4.9 TB/s, what a
// large copy reaches; 88 rows 4.2 us, a launch's latency; append of 11 thousand rows in 8 ragged
// prompts (90 MB) 16.1 to 16.8 us = 5.4 to 5.6 TB/s, of 88 rows 3.4 to 3.6 us.
#include <algorithm>

#include "cs_paged.h"

// ---- argument checks -------------------------------------------------------------------
#define CS_MAX_PSTRIDE ((int64_t)1 << 40)

int cs_check_rows(const char* who, const char* name, const void* base, int64_t row, int64_t head, size_t esz) {
    CS_REQUIRE(base, CS_E_ARG, "%s: %s is NULL", who, name);
    CS_REQUIRE(((uintptr_t)base & 15) == 0, CS_E_ARG, "%s: %s is not aligned to 16 bytes", who, name);
    CS_REQUIRE(row >= 0 && head >= 0 && row <= CS_MAX_PSTRIDE && head <= CS_MAX_PSTRIDE, CS_E_ARG,
               "%s: a stride of %s is negative or too large", who, name);
    CS_REQUIRE(row * esz % 16 == 0 && head * esz % 16 == 0, CS_E_ARG, "%s: a stride of %s is no multiple of 16 bytes", who, name);
    return CS_OK;
}

int cs_check_apart(const char* who, const char* name, int64_t stride0, int64_t n0, int64_t stride1, int64_t n1, int head_dim) {
    CS_REQUIRE((n0 < 2 || stride0 >= head_dim) && (n1 < 2 || stride1 >= head_dim), CS_E_ARG,
               "%s: a stride of %s is less than head_dim: what the call writes would overlap itself", who, name);
    return CS_OK;
}

int cs_check_pages(const char* who, const cs_pages* p) {
    CS_REQUIRE(p, CS_E_ARG, "%s: NULL pages", who);
    CS_REQUIRE(p->dtype == CS_F32 || p->dtype == CS_BF16, CS_E_ARG, "%s: unknown dtype %d", who, p->dtype);
    CS_REQUIRE(p->reserved == 0, CS_E_ARG, "%s: reserved field is not 0", who);
    CS_REQUIRE(p->batch >= 0 && p->n_pages >= 1 && p->n_kv_heads >= 1 && p->table_pages >= 1, CS_E_ARG,
               "%s: a size of the pages is out of range", who);
    CS_REQUIRE(p->batch == 0 || (p->table && p->len), CS_E_ARG, "%s: NULL table or lengths", who);
    CS_REQUIRE(p->table_stride >= p->table_pages, CS_E_ARG, "%s: table_stride is less than table_pages", who);
    CS_REQUIRE(p->head_dim >= 8 && p->head_dim <= 256 && p->head_dim % 8 == 0, CS_E_UNSUPPORTED,
               "%s: head_dim must be a multiple of 8 in 8..256", who);
    CS_REQUIRE(p->page_size >= 16 && p->page_size <= 32768 && (p->page_size & (p->page_size - 1)) == 0, CS_E_UNSUPPORTED,
               "%s: page_size must be a power of two in 16..32768", who);
    CS_REQUIRE((int64_t)p->table_pages * p->page_size <= (int64_t)1 << 30, CS_E_UNSUPPORTED,
               "%s: table_pages * page_size exceeds 2^30", who);
    CS_REQUIRE(p->batch <= 65536 && p->n_kv_heads <= 4096, CS_E_UNSUPPORTED, "%s: too many streams or heads", who);
    const size_t esz = p->dtype == CS_BF16 ? 2 : 4;
    const int64_t page[2] = {p->k_page, p->v_page}, head[2] = {p->k_head, p->v_head}, token[2] = {p->k_token, p->v_token};
    for (int i = 0; i < 2; ++i) {
        CS_TRY(cs_check_rows(who, i ? "v pool" : "k pool", i ? p->v : p->k, page[i], head[i], esz));
        CS_REQUIRE(token[i] >= p->head_dim && token[i] * esz % 16 == 0, CS_E_ARG, "%s: bad token stride", who);
        CS_REQUIRE(token[i] <= (int64_t)0x7fffffff / (int64_t)esz / p->page_size, CS_E_UNSUPPORTED,
                   "%s: a page spans 2^31 bytes or more", who);
    }
    return CS_OK;
}

int cs_pages_view(const char* who, const cs_pages* p, const int32_t* d_row0, int32_t R, cs_pages_dev* d) {
    CS_REQUIRE(R >= 0 && R <= 1 << 26, CS_E_ARG, "%s: R out of range", who);
    CS_REQUIRE(d_row0 || p->batch == 0 || R % p->batch == 0, CS_E_ARG, "%s: R rows cannot be shared out among %d streams without d_row0", who,
               p->batch);
    d->p = *p;
    d->page_log2 = 31 - __builtin_clz((unsigned)p->page_size);
    d->cap = p->table_pages * p->page_size;
    d->row0 = d_row0;
    d->rows = !d_row0 && p->batch ? R / p->batch : 0;
    d->R = R;
    return CS_OK;
}

// ---- one head's elements in a lane ------------------------------------------------------
// VEC elements of either half.  Element pairs of the rotated part are (j, j + rot/2); the part behind
// it is split in two halves the same way and passed through.
template <int VEC>
struct pair_t { float a[VEC], b[VEC]; };

template <int VEC>
__device__ __forceinline__ void ld_vec(const float* p, float* o) {
#pragma unroll
    for (int u = 0; u < VEC; u += 4) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(p + u);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[u + j] = t[j];
    }
}
template <int VEC>
__device__ __forceinline__ void ld_vec(const bf16_t* p, float* o) {
    typedef __bf16 vec __attribute__((ext_vector_type(VEC)));
    const vec t = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int j = 0; j < VEC; ++j) o[j] = (float)t[j];
}
template <int VEC>
__device__ __forceinline__ void st_vec(float* p, const float* v) {
#pragma unroll
    for (int u = 0; u < VEC; u += 4) *reinterpret_cast<f32x4*>(p + u) = (f32x4){v[u], v[u + 1], v[u + 2], v[u + 3]};
}
template <int VEC>
__device__ __forceinline__ void st_vec(bf16_t* p, const float* v) {
    typedef __bf16 vec __attribute__((ext_vector_type(VEC)));
    vec t;
#pragma unroll
    for (int j = 0; j < VEC; ++j) t[j] = (bf16_t)v[j];
    *reinterpret_cast<vec*>(p) = t;
}

// where segment s of a head lies: offsets of the two halves, and the index of its first angle (or -1)
__device__ __forceinline__ void seg_at(int s, int hd, int rot, int vec, int& lo, int& hi, int& ang) {
    const int half = rot >> 1, nrot = half / vec, rest = (hd - rot) >> 1;
    if (s < nrot) {
        lo = s * vec;
        hi = half + lo;
        ang = lo;
    } else {
        lo = rot + (s - nrot) * vec;
        hi = lo + rest;
        ang = -1;
    }
}

template <int VEC>
__device__ __forceinline__ void rotate(pair_t<VEC>& x, const float2* __restrict__ t) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const float2 cs = t[j];
        const float a = x.a[j] * cs.x - x.b[j] * cs.y, b = x.b[j] * cs.x + x.a[j] * cs.y;
        x.a[j] = a;
        x.b[j] = b;
    }
}

// ---- norms and rotation -----------------------------------------------------------------
#define NR_THREADS 256
#define NR_ROWS 4             // most rows of a workgroup
struct nr_side {
    const void* in;
    void* out;
    const float* gain;
    int64_t row, head, out_row, out_head;
};
struct nr_args {
    nr_side s[2];             // queries, keys
    int H, KVH, hd, rot, R, rpw, lanes_log2, segs;
    float eps;
    const int32_t* pos;
    const double* inv_freq;
};

template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(NR_THREADS) void k_qk_norm_rope(nr_args A) {
    __shared__ float2 turn[NR_ROWS * 128];
    const int tid = threadIdx.x;
    const int r0 = (int)cs_paged_wg() * A.rpw, nr = min(A.rpw, A.R - r0), heads = A.H + A.KVH;
    const int seg = tid & ((1 << A.lanes_log2) - 1), per_pass = NR_THREADS >> A.lanes_log2;
    // one task = one head of one row; the heads of a launch's second grid dimension are shared out in turn
    const int n_tasks = nr * heads, first = blockIdx.y * per_pass + (tid >> A.lanes_log2), step = gridDim.y * per_pass;
    int lo, hi, ang;
    seg_at(min(seg, A.segs - 1), A.hd, A.rot, VEC, lo, hi, ang);
    const bool lane_on = seg < A.segs;
    auto request = [&](int t, pair_t<VEC>& x) {
        const int r = t / heads, h = t - r * heads;
        const nr_side& s = A.s[h >= A.H];
        const TI* __restrict__ src = (const TI*)s.in + (int64_t)(r0 + r) * s.row + (int64_t)(h >= A.H ? h - A.H : h) * s.head;
        ld_vec<VEC>(src + lo, x.a);
        ld_vec<VEC>(src + hi, x.b);
    };
    pair_t<VEC> cur, nxt;
    if (first < n_tasks && lane_on) request(first, cur);       // in flight while the angles are made
    const int half = A.rot >> 1;
    for (int i = tid; i < nr * half; i += NR_THREADS) {
        const int r = i / half, j = i - r * half;
        turn[i] = cs_turn(A.pos[r0 + r], A.inv_freq[j]);
    }
    __syncthreads();
    for (int t = first; t < n_tasks; t += step) {
        if (t + step < n_tasks && lane_on) request(t + step, nxt);
        const int r = t / heads, h = t - r * heads;
        const nr_side& s = A.s[h >= A.H];
        if (s.gain) {
            float sq = 0.f;
            if (lane_on)
#pragma unroll
                for (int j = 0; j < VEC; ++j) sq += cur.a[j] * cur.a[j] + cur.b[j] * cur.b[j];
            for (int o = 1 << A.lanes_log2 >> 1; o > 0; o >>= 1) sq += __shfl_xor(sq, o, 64);
            const float inv = 1.0f / sqrtf(sq / (float)A.hd + A.eps);
            if (lane_on) {
                float g[VEC];
                ld_vec<VEC>(s.gain + lo, g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) cur.a[j] *= inv * g[j];
                ld_vec<VEC>(s.gain + hi, g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) cur.b[j] *= inv * g[j];
            }
        }
        if (lane_on) {
            if (ang >= 0) rotate<VEC>(cur, turn + r * half + ang);
            TO* __restrict__ dst = (TO*)s.out + (int64_t)(r0 + r) * s.out_row + (int64_t)(h >= A.H ? h - A.H : h) * s.out_head;
            st_vec<VEC>(dst + lo, cur.a);
            st_vec<VEC>(dst + hi, cur.b);
        }
        cur = nxt;
    }
}

// VEC elements of a half per lane: 8 where rows of 16-bit elements have whole segments of them (16-byte
// loads), else 4
static bool wide_segments(int in_dtype, int hd, int rot) { return in_dtype == CS_BF16 && rot % 16 == 0 && (hd - rot) % 16 == 0; }

static int lanes_log2_of(int segs) {
    int l = 0;
    while (1 << l < segs) ++l;
    return l;
}

static int check_rot(const char* who, const double* inv_freq, int rot, int hd) {
    CS_REQUIRE(rot >= 0 && rot <= hd && rot % 8 == 0, CS_E_ARG, "%s: rot must be a multiple of 8 in 0..head_dim", who);
    CS_REQUIRE(rot == 0 || inv_freq, CS_E_ARG, "%s: NULL inv_freq", who);
    return CS_OK;
}

extern "C" int cs_op_qk_norm_rope(int32_t in_dtype, int32_t out_dtype, const void* q, int64_t q_row, int64_t q_head,
                                  const void* k, int64_t k_row, int64_t k_head, int32_t R, int32_t H, int32_t KVH,
                                  int32_t head_dim, const float* q_gain, const float* k_gain, float eps,
                                  const int32_t* pos, const double* inv_freq, int32_t rot,
                                  void* q_out, int64_t q_out_row, int64_t q_out_head,
                                  void* k_out, int64_t k_out_row, int64_t k_out_head, void* stream) {
    const char* who = "cs_op_qk_norm_rope";
    CS_REQUIRE((in_dtype == CS_F32 && (out_dtype == CS_F32 || out_dtype == CS_BF16)) || (in_dtype == CS_BF16 && out_dtype == CS_BF16),
               CS_E_ARG, "%s: types %d -> %d are not supported", who, in_dtype, out_dtype);
    CS_REQUIRE(R >= 0 && R <= 1 << 26 && H >= 1 && H <= 4096 && KVH >= 0 && KVH <= 4096, CS_E_ARG, "%s: a size is out of range", who);
    CS_REQUIRE(head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0, CS_E_UNSUPPORTED, "%s: head_dim must be a multiple of 8 in 8..256", who);
    CS_TRY(check_rot(who, inv_freq, rot, head_dim));
    CS_REQUIRE(rot == 0 || pos || R == 0, CS_E_ARG, "%s: NULL positions", who);
    CS_REQUIRE(eps >= 0.f && eps <= 1e30f, CS_E_ARG, "%s: eps is negative or not finite", who);
    if (R == 0) return CS_OK;
    const size_t isz = in_dtype == CS_BF16 ? 2 : 4, osz = out_dtype == CS_BF16 ? 2 : 4;
    CS_TRY(cs_check_rows(who, "q", q, q_row, q_head, isz));
    CS_TRY(cs_check_rows(who, "q_out", q_out, q_out_row, q_out_head, osz));
    CS_TRY(cs_check_apart(who, "q_out", q_out_row, R, q_out_head, H, head_dim));
    if (KVH) {
        CS_TRY(cs_check_rows(who, "k", k, k_row, k_head, isz));
        CS_TRY(cs_check_rows(who, "k_out", k_out, k_out_row, k_out_head, osz));
        CS_TRY(cs_check_apart(who, "k_out", k_out_row, R, k_out_head, KVH, head_dim));
    }
    CS_REQUIRE((((uintptr_t)q_gain | (uintptr_t)(KVH ? k_gain : nullptr)) & 15) == 0, CS_E_ARG, "%s: gains are not aligned to 16 bytes", who);
    nr_args A;
    A.s[0] = {q, q_out, q_gain, q_row, q_head, q_out_row, q_out_head};
    A.s[1] = {k, k_out, k_gain, k_row, k_head, k_out_row, k_out_head};
    A.H = H, A.KVH = KVH, A.hd = head_dim, A.rot = rot, A.R = R, A.eps = eps, A.pos = pos, A.inv_freq = inv_freq;
    const bool wide = wide_segments(in_dtype, head_dim, rot);
    A.segs = head_dim / (wide ? 16 : 8);
    A.lanes_log2 = lanes_log2_of(A.segs);
    // The angles of a row are made by every workgroup that has heads of it, and a workgroup has its
    // start and its loads to wait for: one row while there are few, four where they fill the chip
    // several times over, and two workgroups for the heads of a row where one would pass over them more
    // than once (88 rows of 40 heads: 4.6 -> 3.7 us with two; 4096 rows by fours 21.0 -> 17.7).  With
    // one, two and four rows a workgroup, us of captured calls:
    //                             512 rows           1531               2048               4096
    //   40 x 128, bfloat16    5.0   5.4   6.8    9.2   8.6   9.4   11.3  10.3  10.8   18.7  17.2  16.7
    //   32 x 128, bfloat16    4.3   5.4   7.7    7.5   8.2   9.9    8.8   9.3  10.5   15.3  14.6  15.7
    //   32 x 128, float32     5.1   5.9   7.5   10.2  10.0  10.7   13.2  12.3  12.4   22.3  22.2  21.3
    //    9 x 64, bfloat16     3.5   3.4   3.5    4.1   3.9   3.8    4.3   4.0   3.9    6.4   5.2   4.7
    //   32 x 256, bfloat16    6.9   7.3   9.7   14.5  14.7  16.0   16.9  17.5  18.4   26.6  27.8  27.8
    // The rule goes by the rows alone and is the best of the three or within 10 % of it, but around
    // 2048 rows (32 bfloat16 heads of 128: 19 %, 9 float32 heads of 64: 15 %).
    A.rpw = R >= 2048 ? NR_ROWS : R >= 1024 ? 2 : 1;
    const dim3 grid = cs_paged_grid(cs_ceil_div(R, A.rpw), H + KVH > NR_THREADS >> A.lanes_log2 ? 2 : 1);
    hipStream_t s = (hipStream_t)stream;
    if (in_dtype == CS_BF16 && wide) k_qk_norm_rope<bf16_t, bf16_t, 8><<<grid, NR_THREADS, 0, s>>>(A);
    else if (in_dtype == CS_BF16) k_qk_norm_rope<bf16_t, bf16_t, 4><<<grid, NR_THREADS, 0, s>>>(A);
    else if (out_dtype == CS_BF16) k_qk_norm_rope<float, bf16_t, 4><<<grid, NR_THREADS, 0, s>>>(A);
    else k_qk_norm_rope<float, float, 4><<<grid, NR_THREADS, 0, s>>>(A);
    return cs_launch_ok("k_qk_norm_rope");
}

// ---- append -------------------------------------------------------------------------------
struct ap_args {
    const void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    int rot, rpw, lanes_log2, segs;
    const double* inv_freq;
};
// stream of row r: as many streams end at or before it (a wave counts them together, 64 at a time: with a
// row each 1024 streams take 7.6 us, 4096 14.7, 16384 87; without offsets 6.6, 6.7 and 7.4)
__device__ __forceinline__ int stream_of_row(const cs_pages_dev& D, int r) {
    if (!D.row0) return r / D.rows;
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int b0 = 0; b0 < D.p.batch; b0 += 64) {
        const bool ended = b0 + lane < D.p.batch && D.row0[b0 + lane + 1] <= r;
        const int n = __popcll(__ballot(ended));
        b += n;
        if (n < 64) break;
    }
    return b;                                   // batch: a row behind the last stream
}

template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(NR_THREADS) void k_paged_append(cs_pages_dev D, ap_args A) {
    __shared__ float2 turn[NR_ROWS * 128];
    __shared__ int2 dest[NR_ROWS];              // (page, position) of a row, page -1: nowhere
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r0 = (int)cs_paged_wg() * A.rpw, nr = min(A.rpw, D.R - r0), KVH = D.p.n_kv_heads, heads = 2 * KVH;
    const int seg = tid & ((1 << A.lanes_log2) - 1), per_pass = NR_THREADS >> A.lanes_log2;
    const int n_tasks = nr * heads, first = blockIdx.y * per_pass + (tid >> A.lanes_log2), step = gridDim.y * per_pass;
    int lo, hi, ang;
    seg_at(min(seg, A.segs - 1), D.p.head_dim, A.rot, VEC, lo, hi, ang);
    const bool lane_on = seg < A.segs;
    for (int i = wave; i < nr; i += NR_THREADS / CS_WAVE) {
        const int r = r0 + i, b = stream_of_row(D, r);
        int page = -1, pos = 0;
        if (b < D.p.batch) {
            const int2 sr = cs_stream_rows(D, b);
            const int64_t at = (int64_t)cs_stream_len(D, b) + (r - sr.x);
            if (r >= sr.x && r - sr.x < sr.y && at < D.cap) {
                pos = (int)at;
                page = D.p.table[b * D.p.table_stride + (pos >> D.page_log2)];
                if (page < 0 || page >= D.p.n_pages) page = -1;
            }
        }
        if (lane == 0) dest[i] = make_int2(page, pos);
    }
    __syncthreads();
    const int half = A.rot >> 1;
    for (int i = tid; i < nr * half; i += NR_THREADS) {
        const int r = i / half, j = i - r * half;
        turn[i] = cs_turn(dest[r].y, A.inv_freq[j]);
    }
    __syncthreads();
    for (int t = first; t < n_tasks; t += step) {
        const int r = t / heads, h = t - r * heads, g = h < KVH ? h : h - KVH;
        const int2 at = dest[r];
        if (at.x < 0 || !lane_on) continue;
        const bool is_v = h >= KVH;
        const TI* __restrict__ src = is_v ? (const TI*)A.v + (int64_t)(r0 + r) * A.v_row + (int64_t)g * A.v_head
                                          : (const TI*)A.k + (int64_t)(r0 + r) * A.k_row + (int64_t)g * A.k_head;
        pair_t<VEC> x;
        ld_vec<VEC>(src + lo, x.a);
        ld_vec<VEC>(src + hi, x.b);
        if (!is_v && ang >= 0) rotate<VEC>(x, turn + r * half + ang);
        const int slot = at.y & (D.p.page_size - 1);
        TO* __restrict__ dst = is_v ? (TO*)D.p.v + at.x * D.p.v_page + g * D.p.v_head + slot * D.p.v_token
                                    : (TO*)D.p.k + at.x * D.p.k_page + g * D.p.k_head + slot * D.p.k_token;
        st_vec<VEC>(dst + lo, x.a);
        st_vec<VEC>(dst + hi, x.b);
    }
}

extern "C" int cs_paged_append(const cs_pages* p, int32_t src_dtype, const void* k, int64_t k_row, int64_t k_head,
                               const void* v, int64_t v_row, int64_t v_head, const int32_t* d_row0, int32_t R,
                               const double* inv_freq, int32_t rot, void* stream) {
    const char* who = "cs_paged_append";
    CS_TRY(cs_check_pages(who, p));
    CS_REQUIRE(src_dtype == CS_F32 || (src_dtype == CS_BF16 && p->dtype == CS_BF16), CS_E_ARG, "%s: rows of type %d into a cache of type %d",
               who, src_dtype, p->dtype);
    CS_TRY(check_rot(who, inv_freq, rot, p->head_dim));
    cs_pages_dev D;
    CS_TRY(cs_pages_view(who, p, d_row0, R, &D));
    if (R == 0 || p->batch == 0) return CS_OK;
    const size_t isz = src_dtype == CS_BF16 ? 2 : 4;
    CS_TRY(cs_check_rows(who, "k", k, k_row, k_head, isz));
    CS_TRY(cs_check_rows(who, "v", v, v_row, v_head, isz));
    CS_TRY(cs_check_apart(who, "k pool", p->k_page, p->n_pages, p->k_head, p->n_kv_heads, p->head_dim));
    CS_TRY(cs_check_apart(who, "v pool", p->v_page, p->n_pages, p->v_head, p->n_kv_heads, p->head_dim));
    ap_args A = {k, v, k_row, k_head, v_row, v_head, rot, 1, 0, 0, inv_freq};
    const bool wide = wide_segments(src_dtype, p->head_dim, rot);
    A.segs = p->head_dim / (wide ? 16 : 8);
    A.lanes_log2 = lanes_log2_of(A.segs);
    // four rows share the look-up of their places, which is a chain of three loads (11 thousand rows of
    // 8 heads of 128: 19.3 us with one row, 14.4 with four, of 4 heads of 64 13.7 and 7.9; 2048 rows
    // 5.4 and 5.5); few rows are better spread out (88 rows: 3.4 with one, 4.3 with four)
    A.rpw = R >= 1024 ? NR_ROWS : 1;
    const dim3 grid = cs_paged_grid(cs_ceil_div(R, A.rpw));
    hipStream_t s = (hipStream_t)stream;
    if (src_dtype == CS_BF16 && wide) k_paged_append<bf16_t, bf16_t, 8><<<grid, NR_THREADS, 0, s>>>(D, A);
    else if (src_dtype == CS_BF16) k_paged_append<bf16_t, bf16_t, 4><<<grid, NR_THREADS, 0, s>>>(D, A);
    else if (p->dtype == CS_BF16) k_paged_append<float, bf16_t, 4><<<grid, NR_THREADS, 0, s>>>(D, A);
    else k_paged_append<float, float, 4><<<grid, NR_THREADS, 0, s>>>(D, A);
    return cs_launch_ok("k_paged_append");
}
