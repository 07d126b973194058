// Device view of a paged cache, shared by the kernels that fill it and the kernels that read it.
#pragma once

#include "cs_common.h"

// The pages of a cache with what the kernels want precomputed.  An index that comes out of device
// memory (length, row offset, page) is brought into range here before anything is addressed with it.
struct cs_pages_dev {
    cs_pages p;
    int page_log2;
    int cap;                 // positions a stream can have: table_pages * page_size
    const int32_t* row0;     // or NULL: `rows` each
    int rows, R;
};

// first row of stream b and its number of rows, kept inside the R rows of the call
__device__ __forceinline__ int2 cs_stream_rows(const cs_pages_dev& d, int b) {
    if (!d.row0) return make_int2(b * d.rows, d.rows);
    const int a = min(max(d.row0[b], 0), d.R), e = min(max(d.row0[b + 1], 0), d.R);
    return make_int2(a, max(e - a, 0));
}
__device__ __forceinline__ int cs_stream_len(const cs_pages_dev& d, int b) { return min(max(d.p.len[b], 0), d.cap); }

// A launch takes fewer than 2^32 threads along a dimension of its grid: workgroups from 2^CS_GRID_LOG2
// on (512 threads: 2^31) stand along z. Numbers past the last one come up there, and have no work.
#define CS_GRID_LOG2 22
static inline dim3 cs_paged_grid(int64_t n, unsigned y = 1) {
    return n >> CS_GRID_LOG2 ? dim3(1u << CS_GRID_LOG2, y, (unsigned)cs_ceil_div(n, 1 << CS_GRID_LOG2)) : dim3((unsigned)n, y);
}
__device__ __forceinline__ unsigned cs_paged_wg() { return blockIdx.x | blockIdx.z << CS_GRID_LOG2; }

// cos and sin of pos * inv_freq.  The angle is formed in turns in float64 and reduced there to an
// eighth of a turn around the nearest quarter, so far positions lose nothing (at position 2^20 the
// float32 product would be off by 1/16 rad); what is left goes through the Taylor series in float32,
// whose first dropped terms are 1.8e-9 (sine, x^11/11! at pi/4) and 1.2e-10 (cosine, x^12/12!).
__device__ __forceinline__ float2 cs_turn(int pos, double inv_freq) {
    double u = (double)pos * (inv_freq * 0.15915494309189533577);
    const double n = rint(4.0 * u);
    const float x = (float)((u - 0.25 * n) * 6.2831853071795864769);
    const float x2 = x * x;
    const float s = x + x * x2 * (-1.6666667e-1f + x2 * (8.3333333e-3f + x2 * (-1.9841270e-4f + x2 * 2.7557319e-6f)));
    const float c = 1.0f + x2 * (-0.5f + x2 * (4.1666667e-2f + x2 * (-1.3888889e-3f + x2 * (2.4801587e-5f - x2 * 2.7557319e-7f))));
    const int quarter = (int)(n - 4.0 * floor(0.25 * n));
    const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss);
}

int cs_check_pages(const char* who, const cs_pages* p);
// fills d from checked arguments; CS_E_ARG if R rows cannot be shared out
int cs_pages_view(const char* who, const cs_pages* p, const int32_t* d_row0, int32_t R, cs_pages_dev* d);
// strides of what a call writes: n0 rows, pages .. and n1 heads that lie apart (a stride that is never
// taken may be anything)
int cs_check_apart(const char* who, const char* name, int64_t stride0, int64_t n0, int64_t stride1, int64_t n1, int head_dim);
// base pointer and two strides of a tensor of rows of heads
int cs_check_rows(const char* who, const char* name, const void* base, int64_t row, int64_t head, size_t esz);
