// Decode attention over the paged 4-bit cache: one new query per query head, lengths of their own for every unit.
//   o = sum_j softmax_j(scale * q . k_j) v_j,   k_j, v_j: rows of e2m1 codes times their groups' scales
#pragma once
#include "common.cuh"
#include "nibble_cache.cuh"
#include "tc_common.cuh"

namespace flowmm {
namespace nibble {

struct AttnArgs {
    const void *q;                     // [U, Hq, D] dense
    const uint8_t *k, *v;              // pages [n_pages, Hkv, page, D / 2]
    const uint8_t *k_scale, *v_scale;  // [n_pages, Hkv, page, D / 16]
    const int *table, *rows;           // [U, max_pages], [U]
    void *out;                         // [U, Hq, D]
    int *status;
    int U, Hq, Hkv, G, page_shift, n_pages, max_pages;
    float scale_log2;
};

constexpr float kLowest = -3.402823466e38f;

template <typename T> __device__ __forceinline__ float as_float(T x);
template <> __device__ __forceinline__ float as_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// A block has one (unit, query head), its warps every kWarps-th key, a lane D / 32 channels.
constexpr int kSimpleWarps = 8;
template <typename T, int D>
__global__ void __launch_bounds__(kSimpleWarps * 32) nibble_attention_kernel(const AttnArgs A) {
    constexpr int V = D / 32;
    __shared__ float rec[kSimpleWarps][D + 2];
    predecessor_done();
    successor_may_start();
    const int lane = lane_id(), warp = threadIdx.x >> 5, u = blockIdx.x / A.Hq, g = blockIdx.x - u * A.Hq, h = g / A.G;
    int n = A.rows[u];
    const int most = A.max_pages << A.page_shift;
    if ((n < 0 || n > most) && threadIdx.x == 0) report(A.status, kStatusIndex);
    n = max(0, min(n, most));
    float q[V], acc[V], m = kLowest, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        q[i] = A.scale_log2 * as_float(static_cast<const T *>(A.q)[((int64_t)blockIdx.x) * D + lane * V + i]);
        acc[i] = 0.f;
    }
    for (int key = warp; key < n; key += kSimpleWarps) {
        int id = A.table[(int64_t)u * A.max_pages + (key >> A.page_shift)];
        if ((unsigned)id >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); id = 0; }
        const int64_t at = (((int64_t)id * A.Hkv + h) << A.page_shift) + (key & ((1 << A.page_shift) - 1));
        const int word = lane * V / 8, first = lane * V % 8;
        float k[8], v[8], z = 0.f;
        values8(*reinterpret_cast<const uint32_t *>(A.k + at * (D / 2) + word * 4), A.k_scale[at * (D / kGroup) + word / 2], k);
        values8(*reinterpret_cast<const uint32_t *>(A.v + at * (D / 2) + word * 4), A.v_scale[at * (D / kGroup) + word / 2], v);
        float kk[V], vv[V];
#pragma unroll
        for (int c = 0; c < 8; c += V)
            if (first == c)
#pragma unroll
                for (int i = 0; i < V; ++i) { kk[i] = k[c + i]; vv[i] = v[c + i]; }
#pragma unroll
        for (int i = 0; i < V; ++i) z = fmaf(q[i], kk[i], z);
        z = warp_sum(z);
        const float top = fmaxf(m, z), corr = tc::ex2(m - top), p = tc::ex2(z - top);
        l = fmaf(l, corr, p);
        m = top;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(acc[i], corr, p * vv[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) rec[warp][lane * V + i] = acc[i];
    if (lane == 0) { rec[warp][D] = m; rec[warp][D + 1] = l; }
    __syncthreads();
    if (threadIdx.x < D) {
        float top = kLowest, sum = 0.f, o = 0.f;
        for (int w = 0; w < kSimpleWarps; ++w) top = fmaxf(top, rec[w][D]);
        for (int w = 0; w < kSimpleWarps; ++w) {
            const float c = tc::ex2(rec[w][D] - top);
            sum = fmaf(rec[w][D + 1], c, sum);
            o = fmaf(rec[w][threadIdx.x], c, o);
        }
        static_cast<T *>(A.out)[(int64_t)blockIdx.x * D + threadIdx.x] = from_float<T>(n == 0 ? 0.f : o / sum);
    }
}

}  // namespace nibble
}  // namespace flowmm
