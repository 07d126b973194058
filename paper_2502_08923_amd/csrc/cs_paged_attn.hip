// Attention of a chunk of new rows per stream over the pages of its cache (Sec. 3.2: the draft is appended to the context
// and evaluated in one pass; App. B.2: per-layer K, V).
//
//   out[r][h] = sum_t p_t v[t] / sum_t p_t,   p_t = exp(scale * q[r][h] . k[t] - max),   t <= L_b + i, t > L_b + i - window
//
// One pass over the tokens with the running maximum and sum of the softmax in float32.
#include <algorithm>
#include <cmath>

#include "cs_paged.h"

struct pa_args {
    const void* q;
    int64_t q_row, q_head;
    void* out;
    int64_t out_row, out_head;
    int H, G, window;
    float scale2;             // scale * log2(e): scores in base-2 units
};

__device__ __forceinline__ float ld1(const float* p) { return *p; }
__device__ __forceinline__ float ld1(const bf16_t* p) { return (float)*p; }

// a wave per (row, query head): a token per lane for the scores, four features per lane for the output
template <typename T>
__global__ __launch_bounds__(256) void k_paged_plain(cs_pages_dev D, pa_args A) {
    __shared__ float sq[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t task = (int64_t)blockIdx.x * 4 + wave;
    const int hd = D.p.head_dim;
    const int r = (int)(task / A.H), h = (int)(task % A.H), g = h / A.G;
    int b = -1, i = 0;
    if (r < D.R)
        for (int s = 0; s < D.p.batch; ++s) {
            const int2 sr = cs_stream_rows(D, s);
            if (r >= sr.x && r < sr.x + sr.y) { b = s; i = r - sr.x; break; }
        }
    if (b >= 0)
        for (int d = lane; d < hd; d += 64) sq[wave][d] = ld1((const T*)A.q + r * A.q_row + h * A.q_head + d);
    __syncthreads();
    if (b < 0) return;
    const int L = cs_stream_len(D, b);
    const int last = min(L + i, D.cap - 1), first = A.window ? max(0, L + i - A.window + 1) : 0;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = first & ~63; t0 <= last; t0 += 64) {
        const int t = t0 + lane;
        int page = -1;
        float s = -INFINITY;
        if (t >= first && t <= last) {
            page = D.p.table[b * D.p.table_stride + (t >> D.page_log2)];
            if (page >= D.p.n_pages) page = -1;
        }
        const int slot = t & (D.p.page_size - 1);
        if (page >= 0) {
            const T* kr = (const T*)D.p.k + page * D.p.k_page + g * D.p.k_head + slot * D.p.k_token;
            s = 0.f;
            for (int d = 0; d < hd; ++d) s += sq[wave][d] * ld1(kr + d);
            s *= A.scale2;
        }
        const float mn = fmaxf(m, cs_wave_max(s));
        if (mn == -INFINITY) continue;
        const float alpha = exp2f(m - mn), p = page >= 0 ? exp2f(s - mn) : 0.f;
        l = l * alpha + cs_wave_sum(p);
        m = mn;
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] *= alpha;
        for (int j = 0; j < 64; ++j) {
            const int pj = __shfl(page, j, 64);
            const float w = __shfl(p, j, 64);
            if (pj < 0) continue;
            const T* vr = (const T*)D.p.v + pj * D.p.v_page + g * D.p.v_head + ((t0 + j) & (D.p.page_size - 1)) * D.p.v_token;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (lane + 64 * u < hd) o[u] += w * ld1(vr + lane + 64 * u);
        }
    }
    T* out = (T*)A.out + r * A.out_row + h * A.out_head;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (lane + 64 * u < hd) cs_st(out, lane + 64 * u, l > 0.f ? o[u] / l : 0.f);
}

// ---- entry points --------------------------------------------------------------------------
static int check_shape(const char* who, const cs_pages* p, int32_t n_heads, int32_t R, int32_t max_rows, int64_t max_len) {
    CS_TRY(cs_check_pages(who, p));
    CS_REQUIRE(n_heads >= 1 && n_heads <= 4096 && n_heads % p->n_kv_heads == 0, CS_E_ARG,
               "%s: n_heads must be a multiple of n_kv_heads, up to 4096", who);
    CS_REQUIRE(R >= 0 && R <= 1 << 26, CS_E_ARG, "%s: R out of range", who);
    CS_REQUIRE((int64_t)R * n_heads <= 0x7fffffff, CS_E_UNSUPPORTED, "%s: more than 2^31 - 1 query rows", who);
    CS_REQUIRE(max_rows >= 0 && max_len >= 0, CS_E_ARG, "%s: negative max_rows or max_len", who);
    return CS_OK;
}

extern "C" int64_t cs_paged_attention_workspace(const cs_pages* p, int32_t n_heads, int32_t has_row0, int32_t R, int32_t max_rows,
                                                int64_t max_len) {
    const char* who = "cs_paged_attention_workspace";
    CS_TRY(check_shape(who, p, n_heads, R, max_rows, max_len));
    CS_REQUIRE(has_row0 || p->batch == 0 || R % p->batch == 0, CS_E_ARG, "%s: R rows cannot be shared out among %d streams without d_row0",
               who, p->batch);
    return 0;
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
    pa_args A = {q, q_row, q_head, out, out_row, out_head, n_heads, n_heads / p->n_kv_heads, window, scale * 1.4426950408889634f};
    hipStream_t s = (hipStream_t)stream;
    const unsigned grid = (unsigned)cs_ceil_div((int64_t)R * n_heads, 4);
    if (p->dtype == CS_BF16) k_paged_plain<bf16_t><<<grid, 256, 0, s>>>(D, A);
    else k_paged_plain<float><<<grid, 256, 0, s>>>(D, A);
    return cs_launch_ok("k_paged_plain");
}
