// Decode attention over the paged 8-bit cache: one new query per query head, lengths of their own for every unit.
//   o = sum_j softmax_j(scale * q . (sk_j k_j)) (sv_j v_j),   k_j, v_j: e4m3 codes, sk_j, sv_j: their page's scales
// This file: how a call is cut into ranges of keys on the device, where alone the lengths are known, how the ranges of a head are
// joined, and the SIMT kernel (fp32 queries, heads of 64).
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"
#include "tc_common.cuh"

namespace flowmm {
namespace paged {

struct AttnArgs {
    const void *q;                     // [U, Hq, D] dense
    const uint8_t *k, *v;              // pages [n_pages, Hkv, page, D]
    const float *k_scale, *v_scale;    // [n_pages, Hkv]
    const int *table, *rows;           // [U, max_pages], [U]
    float *out;                        // [U, Hq, D]
    float *part;                       // [blocks][G][D + 2]: output relative to the maximum, maximum (log2), sum of weights
    unsigned long long *ticket;        // [U * Hkv * groups]: (call, ranges done)
    int *status;
    uint32_t call;
    int U, Hq, Hkv, G, groups, page, page_shift, n_pages, max_pages, q_bf16;
    int target;                        // ranges in all that the call is cut into, about
    float scale_log2;
};

constexpr float kLowest = -3.402823466e38f;   // where maxima start: no logit is below it, and what it is subtracted from stays a number or -inf

// ---- ranges --------------------------------------------------------------------------------------
// The work of a call is cut by the lengths: tiles of kKeys keys, `per` of them to a range, so that all units together make about
// `target` ranges of equal length (a unit's last one is what remains; a unit without rows has one, which writes zeros).  Every
// block finds its own range: a sum over the units, then the prefix sum until its number falls into a unit.  Ranges are numbered
// by unit, range, then head, so there are at most target + U * heads of them, the blocks of the launch.
struct Range { int u, h, split, n_split, tile0, tiles, rows; };
template <int kThreads> struct RangeScratch { unsigned long long sums[kThreads / 32 + 1]; int scan[33]; Range found; int hit; };

__device__ __forceinline__ int unit_rows(const AttnArgs &A, int u) {
    const int n = A.rows[u], most = A.max_pages << A.page_shift;
    return n < 0 ? 0 : min(n, most);
}

template <int kThreads, int kKeys>
__device__ __forceinline__ bool find_range(const AttnArgs &A, int heads, uint32_t item, RangeScratch<kThreads> &s, Range &r) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long tiles = 0;
    for (int u = tid; u < A.U; u += kThreads) {
        const int n = A.rows[u];
        if (blockIdx.x == 0 && (n < 0 || n > A.max_pages << A.page_shift)) report(A.status, kStatusIndex);
        tiles += (unit_rows(A, u) + kKeys - 1) / kKeys;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) tiles += __shfl_xor_sync(0xFFFFFFFFu, tiles, o);
    if (lane == 0) s.sums[warp] = tiles;
    if (tid == 0) s.hit = 0;
    __syncthreads();
    tiles = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) tiles += s.sums[w];
    const unsigned long long per_all = (tiles * heads + A.target - 1) / A.target;
    const int per = per_all < 1 ? 1 : (int)per_all;
    const uint32_t want = item / heads;
    uint32_t before = 0;
    for (int u0 = 0; u0 < A.U; u0 += kThreads) {
        const int u = u0 + tid;
        const int n = u < A.U ? unit_rows(A, u) : 0, t = (n + kKeys - 1) / kKeys;
        const int mine = u < A.U ? max(1, (t + per - 1) / per) : 0;
        int total;
        const uint32_t at = before + block_exclusive_scan(mine, s.scan, total);
        if (u < A.U && want >= at && want < at + mine) {
            const int split = want - at;
            s.found = {u, (int)(item % heads), split, mine, split * per, min(per, t - split * per), n};
            s.hit = 1;
        }
        before += total;
        if (want < before) break;                                     // (the same for the whole block)
    }
    __syncthreads();
    if (!s.hit) return false;
    r = s.found;
    return true;
}

// ---- joining -------------------------------------------------------------------------------------
// A block that has written its range's record takes a ticket of its head; the one that takes the last joins the records.  The
// ticket carries the call's number, so the memory may hold anything before, and is back at zero after the last one.
__device__ __forceinline__ bool take_ticket(unsigned long long *ticket, uint32_t call, int n) {
    unsigned long long seen = *reinterpret_cast<volatile unsigned long long *>(ticket);
    for (int tries = 0; tries < n; ++tries) {                         // (a lost exchange is another block's ticket: n - 1 at most)
        const uint32_t done = (uint32_t)(seen >> 32) == call ? (uint32_t)seen + 1u : 1u;
        const bool last = done >= (uint32_t)n;
        const unsigned long long prev = atomicCAS(ticket, seen, (unsigned long long)call << 32 | (last ? 0u : done));
        if (prev == seen) return last;
        seen = prev;
    }
    return false;
}

// Joins the records of one head's ranges, `step` floats apart: by heads and dims over the block's threads.
template <int kThreads, int D>
__device__ __forceinline__ void join_ranges(const float *rec, int64_t step, int n, int G, float *out) {
    for (int i = threadIdx.x; i < G * D; i += kThreads) {
        const int g = i / D, d = i % D;
        const float *p = rec + g * (D + 2);
        float mx = kLowest, o = 0.f, l = 0.f;
#pragma unroll 8
        for (int s = 0; s < n; ++s) mx = fmaxf(mx, __ldcg(p + s * step + D));
#pragma unroll 8
        for (int s = 0; s < n; ++s) {
            const float w = tc::ex2(__ldcg(p + s * step + D) - mx);
            o = fmaf(__ldcg(p + s * step + d), w, o);
            l = fmaf(__ldcg(p + s * step + D + 1), w, l);
        }
        out[g * D + d] = o / l;
    }
}

// ---- SIMT ----------------------------------------------------------------------------------------
constexpr int kSimtThreads = 128, kSimtKeys = 64, kSimtPages = 256;

// A group of D / 16 lanes shares a row (16 codes a lane); the groups of a block take the range's keys in turn, kStep rows each with
// K and V on their way at once.  GP: query heads of a range, 1, 2 or 4 (more of a KV head are ranges of their own).
template <int D, int GP>
__global__ void __launch_bounds__(kSimtThreads) cache_attention_kernel(const AttnArgs A) {
    constexpr int kLanes = D / 16, kGroups = kSimtThreads / kLanes, kStep = 2;
    __shared__ RangeScratch<kSimtThreads> scratch;
    __shared__ float rec[kGroups][GP][D + 2];
    __shared__ int ids[kSimtPages];
    __shared__ float ks[kSimtPages], vs[kSimtPages];
    __shared__ int last;
    predecessor_done();
    successor_may_start();
    Range r;
    const int heads = A.Hkv * A.groups;
    if (!find_range<kSimtThreads, kSimtKeys>(A, heads, blockIdx.x, scratch, r)) return;
    const int tid = threadIdx.x, sub = tid % kLanes, grp = tid / kLanes;
    const int h = r.h / A.groups, g0 = (r.h % A.groups) * GP, G = min(GP, A.G - g0);
    float *out = A.out + ((int64_t)r.u * A.Hq + h * A.G + g0) * D;
    if (r.rows == 0) {
        for (int i = tid; i < G * D; i += kSimtThreads) out[i] = 0.f;
        return;
    }
    const int lo = r.tile0 * kSimtKeys, hi = min(r.rows, lo + r.tiles * kSimtKeys);
    float q[GP][16], acc[GP][16], m[GP], l[GP];
#pragma unroll
    for (int g = 0; g < GP; ++g) {
        m[g] = kLowest; l[g] = 0.f;
        const int64_t at = ((int64_t)r.u * A.Hq + h * A.G + g0 + min(g, G - 1)) * D + sub * 16;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            acc[g][e] = 0.f;
            q[g][e] = A.scale_log2 * (A.q_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(A.q)[at + e]) : static_cast<const float *>(A.q)[at + e]);
        }
    }
    const int *table = A.table + (int64_t)r.u * A.max_pages;
    const int first_page = lo >> A.page_shift, last_page = (hi - 1) >> A.page_shift;
    for (int p0 = first_page; p0 <= last_page; p0 += kSimtPages) {    // pages whose numbers and scales are in shared memory at once
        __syncthreads();
        for (int j = tid; j < kSimtPages && p0 + j <= last_page; j += kSimtThreads) {
            int id = table[p0 + j];
            if (id < 0 || id >= A.n_pages) { report(A.status, kStatusIndex); id = 0; }
            ids[j] = id;
            ks[j] = A.k_scale[(int64_t)id * A.Hkv + h];
            vs[j] = A.v_scale[(int64_t)id * A.Hkv + h];
        }
        __syncthreads();
        const int from = max(lo, p0 << A.page_shift), to = (int)min((int64_t)hi, (int64_t)(p0 + kSimtPages) << A.page_shift);
        for (int base = from; base < to; base += kGroups * kStep) {   // the same number of steps for every lane group
            uint4 kr[kStep], vr[kStep];
            float kscale[kStep], vscale[kStep];
            const int key0 = base + grp * kStep;
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                const int key = min(key0 + i, to - 1), j = (key >> A.page_shift) - p0;
                const int64_t at = ((((int64_t)ids[j] * A.Hkv + h) << A.page_shift) + (key & (A.page - 1))) * D + sub * 16;
                kr[i] = *reinterpret_cast<const uint4 *>(A.k + at);
                vr[i] = *reinterpret_cast<const uint4 *>(A.v + at);
                kscale[i] = ks[j]; vscale[i] = vs[j];
            }
            float z[kStep][GP];
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                float k[16];
                from_e4m3x16(kr[i], k);
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    float d = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) d = fmaf(q[g][e], k[e], d);
                    z[i][g] = d;
                }
            }
#pragma unroll
            for (int o = kLanes >> 1; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < kStep; ++i)
#pragma unroll
                    for (int g = 0; g < GP; ++g) z[i][g] += __shfl_xor_sync(0xFFFFFFFFu, z[i][g], o);
            float p[kStep][GP];
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                float mx = m[g], add = 0.f;
#pragma unroll
                for (int i = 0; i < kStep; ++i) {
                    z[i][g] *= kscale[i];
                    if (key0 + i < to) mx = fmaxf(mx, z[i][g]);
                }
                const float corr = tc::ex2(m[g] - mx);
#pragma unroll
                for (int i = 0; i < kStep; ++i) {
                    p[i][g] = key0 + i < to ? tc::ex2(z[i][g] - mx) : 0.f;
                    add += p[i][g];
                    p[i][g] *= vscale[i];
                }
                l[g] = l[g] * corr + add;
                m[g] = mx;
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[g][e] *= corr;
            }
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                float v[16];
                from_e4m3x16(vr[i], v);
#pragma unroll
                for (int g = 0; g < GP; ++g)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[g][e] = fmaf(p[i][g], v[e], acc[g][e]);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GP; ++g) {
#pragma unroll
        for (int e = 0; e < 16; ++e) rec[grp][g][sub * 16 + e] = acc[g][e];
        if (sub == 0) { rec[grp][g][D] = m[g]; rec[grp][g][D + 1] = l[g]; }
    }
    __syncthreads();
    float *part = A.part + (int64_t)blockIdx.x * GP * (D + 2);
    for (int i = tid; i < G * D; i += kSimtThreads) {
        const int g = i / D, d = i % D;
        float mx = kLowest, o = 0.f, ls = 0.f;
        for (int w = 0; w < kGroups; ++w) mx = fmaxf(mx, rec[w][g][D]);
        for (int w = 0; w < kGroups; ++w) {
            const float c = tc::ex2(rec[w][g][D] - mx);
            o = fmaf(rec[w][g][d], c, o);
            ls = fmaf(rec[w][g][D + 1], c, ls);
        }
        if (r.n_split == 1) {
            out[i] = o / ls;
        } else {
            part[g * (D + 2) + d] = o;
            if (d == 0) { part[g * (D + 2) + D] = mx; part[g * (D + 2) + D + 1] = ls; }
        }
    }
    if (r.n_split == 1) return;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = take_ticket(A.ticket + (int64_t)r.u * heads + r.h, A.call, r.n_split);
    __syncthreads();
    if (!last) return;
    __threadfence();
    join_ranges<kSimtThreads, D>(A.part + ((int64_t)blockIdx.x - (int64_t)r.split * heads) * GP * (D + 2), (int64_t)heads * GP * (D + 2), r.n_split, G, out);
}

}  // namespace paged
}  // namespace flowmm
