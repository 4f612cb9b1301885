// Decode attention over the paged 8-bit cache: one new query per query head, lengths of their own for every unit.
//   o = sum_j softmax_j(scale * q . (sk_j k_j)) (sv_j v_j),   k_j, v_j: e4m3 codes, sk_j, sv_j: their page's scales
// This file: how the SIMT kernel's work is cut into ranges of keys on the device, where alone the lengths are known, the kernel that joins
// ranges, and the SIMT kernel (fp32 queries).
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
    float *part;                       // records (record_floats): one for each block, two on the tensor cores
    int *status;
    int4 *cut_heads;                   // [blocks]: unit, first query head, number of records (0: nothing) and query heads of what begins in the
                                       // block and is to be joined; null: nothing can be
    int U, Hq, Hkv, G, groups, page, page_shift, n_pages, max_pages, q_bf16;
    int target;                        // ranges in all that the call is cut into, about
    FastDiv by_heads;                  // by Hkv * groups
    float scale_log2;
};

constexpr float kLowest = -3.402823466e38f;   // where maxima start: no logit is below it, and what it is subtracted from stays a number or -inf

// ---- ranges --------------------------------------------------------------------------------------
// The work of a call is cut by the lengths: tiles of kKeys keys, `per` of them to a range, so that all units together make about
// `target` ranges of equal length (a unit's last one is what remains; a unit without rows has one, which writes zeros).  Where that would
// cut the longest unit for a few tiles only, nothing is cut: joining costs as much as kJoinTiles tiles.  Every warp
// finds its block's range by itself: a sum over the units, then a prefix sum (each lane some consecutive units) until the
// block's number falls into a unit.  Ranges are numbered by unit, range, then head, so there are at most target + U * heads of
// them, the blocks of the launch.  (With the whole block and its barriers 2.0 us for one unit, so 0.6.)
constexpr int kJoinTiles = 4;
struct Range { int u, h, split, n_split, tile0, tiles, rows; };

__device__ __forceinline__ int unit_rows(const AttnArgs &A, int u) {
    const int n = A.rows[u], most = A.max_pages << A.page_shift;
    return n < 0 ? 0 : min(n, most);
}

template <int kKeys>
__device__ __forceinline__ bool find_range(const AttnArgs &A, uint32_t item, Range &r) {
    const int lane = lane_id();
    const uint32_t heads = A.by_heads.d, want = A.by_heads.div(item);
    unsigned long long sum = 0;
    int longest = 0;
#pragma unroll 4
    for (int u = lane; u < A.U; u += 32) {
        const int t = (unit_rows(A, u) + kKeys - 1) / kKeys;
        sum += t;
        longest = max(longest, t);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        longest = max(longest, __shfl_xor_sync(0xFFFFFFFFu, longest, o));
    }
    const unsigned long long tiles = sum * heads + A.target - 1;
    const unsigned long long even = tiles >> 32 ? tiles / A.target : (uint32_t)tiles / (uint32_t)A.target;
    const int per = longest <= (int)even + kJoinTiles ? max(1, longest) : max(1, (int)even);
    const int each = (A.U + 31) >> 5, u0 = min(A.U, lane * each), u1 = min(A.U, u0 + each);
    uint32_t mine = 0;
#pragma unroll 4
    for (int u = u0; u < u1; ++u) mine += max(1u, ((uint32_t)(unit_rows(A, u) + kKeys - 1) / kKeys + per - 1) / (uint32_t)per);
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += x;
    }
    const uint32_t hit = __ballot_sync(0xFFFFFFFFu, want < upto);      // the first lane whose units reach the number
    if (hit == 0) return false;
    const int owner = __ffs(hit) - 1;
    int u = 0, split = 0, n_split = 0, t = 0, rows = 0;
    if (lane == owner) {
        uint32_t at = upto - mine;
        for (u = u0; u < u1; ++u) {
            rows = unit_rows(A, u);
            t = (rows + kKeys - 1) / kKeys;
            n_split = max(1u, ((uint32_t)t + per - 1) / (uint32_t)per);
            if (want < at + n_split) break;
            at += n_split;
        }
        split = want - at;
    }
    r.u = __shfl_sync(0xFFFFFFFFu, u, owner);
    r.split = __shfl_sync(0xFFFFFFFFu, split, owner);
    r.n_split = __shfl_sync(0xFFFFFFFFu, n_split, owner);
    r.rows = __shfl_sync(0xFFFFFFFFu, rows, owner);
    t = __shfl_sync(0xFFFFFFFFu, t, owner);
    r.h = item - want * heads;
    r.tile0 = r.split * per;
    r.tiles = min(per, t - r.tile0);
    return true;
}

// Lengths out of range, reported once a call.
__device__ __forceinline__ void check_lengths(const AttnArgs &A) {
    if (blockIdx.x == 0)
        for (int u = threadIdx.x; u < A.U; u += blockDim.x) {
            const int n = A.rows[u];
            if (n < 0 || n > A.max_pages << A.page_shift) report(A.status, kStatusIndex);
        }
}

// ---- joining -------------------------------------------------------------------------------------
// A range's record: its G heads' outputs, relative to the maximum, then the maxima (log2) and the sums of weights.
__host__ __device__ __forceinline__ int record_floats(int G, int D) { return (G * (D + 2) + 3) & ~3; }

// A warp's part of joining one query head: records first, first + stride, ... below n of its ranges, `step` floats apart (the first range's
// `ahead` floats behind its place), relative to the largest of their maxima.  The maxima and sums are read 32 at once, the outputs eight.
template <int D> struct Joined { float top, sum, o[D / 32]; };
template <int D>
__device__ __forceinline__ Joined<D> join_part(const float *rec, int64_t ahead, int64_t step, int first, int stride, int n, int G, int g) {
    constexpr int V = D / 32;
    const int lane = lane_id(), count = first < n ? (n - first + stride - 1) / stride : 0;
    auto record = [&](int i) { const int s = first + i * stride; return rec + s * step + (s == 0 ? ahead : 0); };
    Joined<D> j;
    j.top = kLowest;
    j.sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) j.o[i] = 0.f;
    for (int i = lane; i < count; i += 32) j.top = fmaxf(j.top, __ldcg(record(i) + G * D + g));
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) j.top = fmaxf(j.top, __shfl_xor_sync(0xFFFFFFFFu, j.top, i));
    for (int i0 = 0; i0 < count; i0 += 32) {
        const bool on = i0 + lane < count;
        const float w = on ? tc::ex2(__ldcg(record(i0 + lane) + G * D + g) - j.top) : 0.f;
        if (on) j.sum = fmaf(__ldcg(record(i0 + lane) + G * D + G + g), w, j.sum);
        for (int i1 = i0; i1 < min(count, i0 + 32); i1 += 8) {
            float x[8][V];
#pragma unroll
            for (int i = 0; i < 8; ++i) {                             // (places past the last range: the last one again, with a weight of zero)
                const float *at = record(min(i1 + i, count - 1)) + g * D + lane * V;
                if (V == 4) {
                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(at));
                    x[i][0] = v.x; x[i][1] = v.y; x[i][V - 2] = v.z; x[i][V - 1] = v.w;
                } else {
                    const float2 v = __ldcg(reinterpret_cast<const float2 *>(at));
                    x[i][0] = v.x; x[i][1] = v.y;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = __shfl_sync(0xFFFFFFFFu, w, (i1 - i0 + i) & 31);
                if (i1 + i < count) {
#pragma unroll
                    for (int k = 0; k < V; ++k) j.o[k] = fmaf(x[i][k], c, j.o[k]);
                }
            }
        }
    }
    j.sum = warp_sum(j.sum);
    return j;
}

// Joins what was cut (AttnArgs::cut_heads), in an order that goes by the ranges' number alone: a block for every block that it can begin in,
// kWarps warps for each query head, with every kWarps-th record each.  A block of the kernel before has `own` records; the first one of a
// join is the `first`-th of its block, the next ones are `step` records apart, counted from its block's first.
// (By the range that ended last, which it learnt from a ticket: 35 ranges that end together drew theirs one after the other, 4 sequences of 2200 rows, 4 heads of 64,
// 22.6 us, so 10.)  Four warps where heads are few, and so cut into many ranges, else one, which makes the blocks that find nothing to do fewer.  The call with
// four and with one, sequences of up to 8448 rows: tensor cores, 4 heads (33 records of each) 12.4 and 14.5 us, 16 heads 14.8 and 15.3, 32 heads 18.4 and
// 18.4, 72 heads 26.6 and 25.5; SIMT, 32 heads 13.2 and 14.3, 64 heads 19.6 and 20.1, 80 heads 24.0 and 23.9.  16 sequences of up to 33 792 rows,
// 8 heads: 108.9 and 107.0.
constexpr int kJoinThreads = 256, kFewHeads = 74;
template <int D, int kWarps>
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(const AttnArgs A, const int record, const int own, const int first, const int step) {
    constexpr int kTeams = kJoinThreads / 32 / kWarps, V = D / 32;
    predecessor_done();
    successor_may_start();
    const int4 cut = A.cut_heads[blockIdx.x];
    const int lane = lane_id(), team = (threadIdx.x >> 5) / kWarps, p = (threadIdx.x >> 5) % kWarps, g = blockIdx.y * kTeams + team, G = cut.w;
    if (cut.z == 0 || g >= G) return;                                 // (whole teams)
    const Joined<D> j = join_part<D>(A.part + (int64_t)blockIdx.x * own * record, (int64_t)first * record, (int64_t)step * record, p, kWarps, cut.z, G, g);
    float *out = A.out + ((int64_t)cut.x * A.Hq + cut.y + g) * D;
    if constexpr (kWarps == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[lane * V + i] = j.o[i] / j.sum;
    } else {
        __shared__ float parts[kTeams][kWarps][D], tops[kTeams][kWarps], sums[kTeams][kWarps];
#pragma unroll
        for (int i = 0; i < V; ++i) parts[team][p][lane * V + i] = j.o[i];
        if (lane == 0) { tops[team][p] = j.top; sums[team][p] = j.sum; }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(kWarps * 32) : "memory");
        float top = kLowest, sum = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) top = fmaxf(top, tops[team][i]);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) sum = fmaf(sums[team][i], tc::ex2(tops[team][i] - top), sum);
        for (int d = p * 32 + lane; d < D; d += kWarps * 32) {
            float o = 0.f;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) o = fmaf(parts[team][i][d], tc::ex2(tops[team][i] - top), o);
            out[d] = o / sum;
        }
    }
}

// ---- SIMT ----------------------------------------------------------------------------------------
constexpr int kSimtThreads = 128, kSimtKeys = 64, kSimtPages = 256;

// A group of D / 16 lanes shares a row (16 codes a lane); the groups of a block take the range's keys in turn, kStep rows each with
// K and V on their way at once.  GP: query heads of a range, 1 or 2; more of a KV head are ranges of their own, which find its rows in L2 (four to a
// range took 212 registers: 8 units of up to 2200 rows, 8 heads of 4 query heads 17.2 us, by two 14.2; 200 units 178 and 171).
template <int D, int GP>
__global__ void __launch_bounds__(kSimtThreads) cache_attention_kernel(const AttnArgs A) {
    constexpr int kLanes = D / 16, kGroups = kSimtThreads / kLanes, kStep = GP == 1 ? 4 : 2;
    __shared__ float rec[kGroups][GP][D + 2];
    __shared__ int ids[kSimtPages];
    __shared__ float ks[kSimtPages], vs[kSimtPages];
    predecessor_done();
    successor_may_start();
    Range r = {};
    check_lengths(A);
    const bool work = find_range<kSimtKeys>(A, blockIdx.x, r);
    if (A.cut_heads && threadIdx.x == 0) {
        const int g0 = (r.h % A.groups) * GP;
        A.cut_heads[blockIdx.x] = work && r.split == 0 && r.n_split > 1 ? make_int4(r.u, r.h / A.groups * A.G + g0, r.n_split, min(GP, A.G - g0))
                                                                         : make_int4(0, 0, 0, 0);
    }
    if (!work) return;
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
    const int record = record_floats(GP, D);
    float *part = A.part + (int64_t)blockIdx.x * record;
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
            part[i] = o;
            if (d == 0) { part[G * D + g] = mx; part[G * D + G + g] = ls; }
        }
    }
}

}  // namespace paged
}  // namespace flowmm
