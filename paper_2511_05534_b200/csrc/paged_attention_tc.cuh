// Decode attention over the paged 8-bit cache on the tensor cores: bf16 queries, heads of 128.
//
// The codes go into the matrix instructions as they are (kind::f8f6f4), with the keys on the wide side, so no code is ever
// converted and every row of K and V is read once.  The narrow side is split into e4m3 numbers that stand side by side as columns:
//   S[key, head]: a bf16 query, scaled by a power of two, is the sum of two e4m3 numbers, 8 bits of significand as 4 + 4 (exact but
//                 for elements 2^13 times smaller than the largest): N = 8 heads x 2
//   O[dim, head]: a weight is kept as four e4m3 numbers, each the rounded rest of the one before times 16, within 2^-16 of
//                 itself: N = 8 heads x 4.  (Two, the error of a bf16 weight, would not shorten anything that bounds: see below.)
// The pages' scales join in fp32: K's on the logits; V's in the exponent of the weights, w_j = 2^(z_j + log2 sv_j - max), with a maximum of
// its own, so that the largest weight is 1 whatever the scales are.  The sum of the softmax, sum_j 2^(z_j - max z), is apart.
//
// A block takes a range of tiles of 128 keys (paged_attention.cuh) of one (unit, KV head), in groups of seven tiles:
//   warp 0     K tiles and V tiles by TMA, a box per page, into a ring of six stages of 16 KB: K of group c + 1 before V of group c
//   warp 1     the products, in the same order; the logits of two groups stay in tensor memory
//   warps 2-9  a thread per key of a tile: maxima of a group, then its weights; a thread per dim: the output, rescaled once a group.
//              Two halves of four warps: for more than four query heads each has four of them, for fewer every other tile.  (One half
//              alone took 1800 clocks for a tile of eight heads, and two such blocks to an SM longer than the memory.)
// Two blocks share an SM (256 columns of tensor memory and 110 KB each).  Every wait is bounded.
#pragma once
#include "paged_attention.cuh"

namespace flowmm {
namespace paged {
namespace ptc {

constexpr int kTile = 128, kStages = 6, kMaxHeads = 8, kHalf = 4, kGroup = 7, kThreads = 320, kTmemCols = 256;
constexpr int kQCols = 2 * kMaxHeads, kPCols = 4 * kMaxHeads;            // N of the two products; by half, piece, head
constexpr int kMostPages = kGroup * kTile / 16;                          // pages of a group
constexpr uint32_t kStageBytes = kTile * 128;
constexpr uint32_t kSmemQ = kStages * kStageBytes, kSmemP = kSmemQ + kQCols * 128, kSmemRed = kSmemP + 2 * kPCols * 128;
constexpr uint32_t kSmemInfo = kSmemRed + 2 * 8 * 2 * kHalf * 4;          // red: [group parity][warp][maxima, with V's scales][head]
constexpr uint32_t kSmemQInv = kSmemInfo + 3 * 2 * kMostPages * 4;        // info: [group mod 3][K's scale, log2 of V's][page]
constexpr uint32_t kSmemBar = kSmemQInv + kMaxHeads * 4;
constexpr int kBarFull = 0, kBarEmpty = kStages, kBarQ = 2 * kStages, kBarS = kBarQ + 1, kBarPFull = kBarS + 2 * kGroup,
              kBarPEmpty = kBarPFull + 2, kBarO = kBarPEmpty + 2, kNumBars = kBarO + 1;
constexpr uint32_t kSmemBytes = kSmemBar + 8 * kNumBars + 16;             // (+ TMEM address, abort flag, status, last)
constexpr uint32_t kColS = kPCols;                                        // O in the first columns, then the two groups' logits
static_assert(kColS + 2 * kGroup * kQCols <= kTmemCols, "tensor memory");
static_assert(2 * (kSmemBytes + 1024) <= 227 * 1024, "two blocks to an SM");

__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N) { return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24); }
constexpr uint32_t kIdescQK = idesc_e4m3(kTile, kQCols);
constexpr uint32_t kIdescPV = 1u << 15;                                   // V with the dims (M) contiguous: a row is one key

// D[tmem] (+)= A[smem] B[smem]^T, e4m3 inputs, fp32 accumulate; one thread issues.
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 a, {%1, %3};\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %4, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(tc::kDescSw128Hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 8 consecutive fp32 columns of this thread's TMEM lane, waited for.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void epi_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void sts8(uint32_t addr, uint32_t v) { asm volatile("st.shared.b8 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float log2_of(float x) {
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x in [0, 256] as four e4m3 numbers, p0 + p1 / 16 + p2 / 256 + p3 / 4096, for two x at once; each piece two codes
__device__ __forceinline__ void four_pieces(float a, float b, uint32_t (&piece)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        piece[i] = to_e4m3x2(a, b);
        if (i == 3) break;
        const float2 f = from_e4m3x2(piece[i]);
        a = (a - f.x) * 16.f;
        b = (b - f.y) * 16.f;
    }
}

// kByTiles: at most four query heads, the halves take every other tile; else the halves have four heads each.
template <bool kByTiles>
__global__ void __launch_bounds__(kThreads, 2)
cache_attention_tc_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttnArgs A) {
    constexpr int kCols = kByTiles ? kPCols / 2 : kPCols;            // N of the second product
    constexpr uint32_t kPv = kIdescPV | idesc_e4m3(128, kCols);
    extern __shared__ __align__(1024) uint8_t ptc_smem[];
    const uint32_t base = tc::smem_u32(ptc_smem), bars = base + kSmemBar;
    const int warp = tc::warp_number(), lane = threadIdx.x & 31;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(ptc_smem + kSmemBar + 8 * kNumBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *cta_status = reinterpret_cast<int *>(tmem_slot + 2);
    volatile int *last = reinterpret_cast<volatile int *>(tmem_slot + 3);
    if ((base & 1023u) != 0) {                       // the swizzled tiles need a 1024-byte aligned base
        predecessor_done();
        if (threadIdx.x == 0) report(A.status, 6);
        return;
    }
    auto bar = [&](int i) { return bars + 8u * i; };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kNumBars; ++i)
            tc::mbar_init(bar(i), i == kBarQ ? 256 : i == kBarPFull || i == kBarPFull + 1 ? (kByTiles ? 128 : 256) : 1);
        *abort_flag = 0;
        *cta_status = 0;
        tc::mbar_init_fence();
        tc::tma_prefetch_desc(&kmap);
        tc::tma_prefetch_desc(&vmap);
    }
    if (warp == 1) tc::tmem_alloc(tc::smem_u32(tmem_slot), kTmemCols);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    predecessor_done();
    successor_may_start();

    Range r;
    check_lengths(A);
    const bool work = find_range<kTile>(A, blockIdx.x, r);
    const int nt = work ? r.tiles : 0, groups = (nt + kGroup - 1) / kGroup;
    const int key0 = work ? r.tile0 * kTile : 0, G = A.G;
    const int *table = A.table + (int64_t)(work ? r.u : 0) * A.max_pages;
    const int page_at = key0 >> A.page_shift, pages = work ? (r.rows + A.page - 1) >> A.page_shift : 0;   // first page of the range; the unit's
    const int tile_pages = kTile >> A.page_shift, record = record_floats<128>(G);
    unsigned long long *ticket = A.ticket + (work ? (int64_t)r.u * A.Hkv + r.h : 0), seen = 0;
    if (threadIdx.x == 32 && work && r.n_split > 1) seen = *reinterpret_cast<volatile unsigned long long *>(ticket);

    if (!work || r.rows == 0) {
        if (work) {
            float *out = A.out + ((int64_t)r.u * A.Hq + r.h * G) * 128;
            for (int i = threadIdx.x; i < G * 128; i += kThreads) out[i] = 0.f;
        }
    } else if (warp == 0) {
        // numbers of a group's pages, two a lane: of the group before, of this one and of the next
        auto numbers = [&](int c, int &a, int &b) {
            const int j = page_at + c * kGroup * tile_pages + lane, end = min(pages, page_at + (c + 1) * kGroup * tile_pages);
            a = j < end ? table[j] : 0;
            b = j + 32 < end ? table[j + 32] : 0;
            if ((unsigned)a >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); a = 0; }
            if ((unsigned)b >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); b = 0; }
        };
        int st = 0, phase = 0;
        auto tiles = [&](const CUtensorMap *m, int c, int a, int b) {
            const int n = min(kGroup, nt - c * kGroup);
            for (int t = 0; t < n; ++t) {
                if (!tc::mbar_wait_warp(bar(kBarEmpty + st), phase ^ 1, abort_flag, cta_status)) return false;
                const int slot = t * tile_pages + lane;
                const int x = __shfl_sync(0xFFFFFFFFu, a, slot & 31), y = __shfl_sync(0xFFFFFFFFu, b, slot & 31), id = slot < 32 ? x : y;
                const int here = min(tile_pages, pages - page_at - (c * kGroup + t) * tile_pages);      // pages of the tile that there are
                if (tc::elect_one()) tc::mbar_expect_tx(bar(kBarFull + st), (uint32_t)here << (A.page_shift + 7));
                __syncwarp();
                if (lane < here) tc::tma_load_4d(base + st * kStageBytes + ((uint32_t)lane << (A.page_shift + 7)), m, bar(kBarFull + st), 0, 0, r.h, id);
                __syncwarp();
                if (++st == kStages) { st = 0; phase ^= 1; }
            }
            return true;
        };
        int before_a = 0, before_b = 0, a, b, next_a = 0, next_b = 0;
        numbers(0, a, b);
        bool ok = true;
        for (int c = 0; ok && c < groups; ++c) {
            if (c + 1 < groups) numbers(c + 1, next_a, next_b);
            ok = tiles(&kmap, c, a, b);
            if (ok && c > 0) ok = tiles(&vmap, c - 1, before_a, before_b);
            before_a = a; before_b = b; a = next_a; b = next_b;
        }
        if (ok) ok = tiles(&vmap, groups - 1, before_a, before_b);
        if (!ok)         // winding down after a timeout: give copies already issued a moment to land
            for (int i = 0; i < kStages; ++i)
                for (int s = 0; s < (1 << 16) && !tc::mbar_try_wait(bar(kBarFull + i), 0) && !tc::mbar_try_wait(bar(kBarFull + i), 1); ++s) {}
    } else if (warp == 1) {
        const uint32_t q_lo = tc::desc_lo(base + kSmemQ);
        int st = 0, phase = 0;
        auto next = [&]() { if (++st == kStages) { st = 0; phase ^= 1; } };
        auto logits = [&](int c) {
            const int n = min(kGroup, nt - c * kGroup);
            for (int t = 0; t < n; ++t, next()) {
                if (!tc::mbar_wait_warp(bar(kBarFull + st), phase, abort_flag, cta_status)) return false;
                tc::tc_fence_after();
                const uint32_t a_lo = tc::desc_lo(base + st * kStageBytes), at = tmem + kColS + ((c & 1) * kGroup + t) * kQCols;
                if (tc::elect_one()) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_e4m3(at, a_lo + 2 * j, q_lo + 2 * j, kIdescQK, j > 0);
                    tc::umma_commit(bar(kBarEmpty + st));
                    tc::umma_commit(bar(kBarS + (c & 1) * kGroup + t));
                }
                __syncwarp();
            }
            return true;
        };
        auto output = [&](int c) {
            const int n = min(kGroup, nt - c * kGroup);
            for (int t = 0; t < n; ++t, next()) {
                const int i = c * kGroup + t, pb = i & 1;
                if (!tc::mbar_wait_warp(bar(kBarFull + st), phase, abort_flag, cta_status) ||
                    !tc::mbar_wait_warp(bar(kBarPFull + pb), (i >> 1) & 1, abort_flag, cta_status))
                    return false;
                tc::tc_fence_after();
                const uint32_t a_lo = tc::desc_lo(base + st * kStageBytes), p_lo = tc::desc_lo(base + kSmemP + pb * kPCols * 128);
                if (tc::elect_one()) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_e4m3(tmem, a_lo + 256 * j, p_lo + 2 * j, kPv, (t | j) != 0);
                    tc::umma_commit(bar(kBarEmpty + st));
                    tc::umma_commit(bar(kBarPEmpty + pb));
                    if (t == n - 1) tc::umma_commit(bar(kBarO));
                }
                __syncwarp();
            }
            return true;
        };
        bool ok = tc::mbar_wait_warp(bar(kBarQ), 0, abort_flag, cta_status);
        for (int c = 0; ok && c < groups; ++c) {
            ok = logits(c);
            if (ok && c > 0) ok = output(c - 1);
        }
        if (ok) output(groups - 1);
    } else {
        const int e = threadIdx.x - 64, half = e >> 7;               // 0 .. 255
        const int row = 32 * (warp & 3) + lane;                      // TMEM lane this thread reads: key of a tile / output dim
        const uint32_t trow = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const int set = kByTiles ? 0 : half, g0 = kHalf * set;       // this half's heads
        const int part_of = kByTiles ? half : 0, parts = kByTiles ? 2 : 1;   // ... and tiles: those with i % parts == part_of
        const uint32_t tcols = trow + set * 8;                       // columns of their logits within a tile's
        float *red = reinterpret_cast<float *>(ptc_smem + kSmemRed), *info = reinterpret_cast<float *>(ptc_smem + kSmemInfo);
        float *qinv = reinterpret_cast<float *>(ptc_smem + kSmemQInv);
        // scales of a group's pages, one a thread
        auto scales = [&](int c, float &k, float &lv) {
            const int j = page_at + c * kGroup * tile_pages + e;
            k = 0.f; lv = 0.f;
            if (e < kGroup * tile_pages && j < pages) {
                int id = table[j];
                if ((unsigned)id >= (unsigned)A.n_pages) id = 0;    // (the loader has reported it)
                k = A.k_scale[(int64_t)id * A.Hkv + r.h];
                lv = log2_of(A.v_scale[(int64_t)id * A.Hkv + r.h]);
            }
        };
        float next_k, next_lv;
        scales(0, next_k, next_lv);
        {   // the query operand: a warp per head (zero beyond G), four elements a lane
            const int g = e >> 5;
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (g < G) {
                const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(A.q) + ((int64_t)r.u * A.Hq + r.h * G + g) * 128 + lane * 4);
                x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
                x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
            }
            float size = 0.f;
            bool fine = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) { size = fmaxf(size, fabsf(x[i])); fine = fine && is_finite(x[i]); }
            if (!fine) size = __uint_as_float(0x7F800000u);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) size = fmaxf(size, __shfl_xor_sync(0xFFFFFFFFu, size, o));
            const int ex = is_finite(size) ? max(-100, (int)(__float_as_uint(size) >> 23) - 127) - 7 : 0;   // the largest element to [128, 256)
            const float f = power_of_two(-ex);
            uint32_t lo[2], hi[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float a = x[2 * i] * f, b = x[2 * i + 1] * f;
                hi[i] = to_e4m3x2(a, b);
                const float2 h = from_e4m3x2(hi[i]);
                lo[i] = to_e4m3x2((a - h.x) * 16.f, (b - h.y) * 16.f);
            }
            // rows of the operand: by half, piece, head
            const int n = (g >> 2) * 8 + (g & 3);
            const uint32_t at = base + kSmemQ + (lane & 3) * 4;
            sts32(at + n * 128 + (((lane >> 2) ^ (n & 7)) << 4), hi[0] | hi[1] << 16);
            sts32(at + (n + 4) * 128 + (((lane >> 2) ^ ((n + 4) & 7)) << 4), lo[0] | lo[1] << 16);
            // a query that is not finite: its logits become NaN by this factor
            if (lane == 0) qinv[g] = is_finite(size) ? power_of_two(ex) * A.scale_log2 : __uint_as_float(0x7FC00000u);
        }
        fence_proxy_async();
        tc::mbar_arrive(bar(kBarQ));
        if (e < kMostPages) { info[e] = next_k; info[kMostPages + e] = next_lv; }
        epi_sync();

        float cq[kHalf], m[kHalf], mv[kHalf], l[kHalf], acc[kHalf];
#pragma unroll
        for (int g = 0; g < kHalf; ++g) { cq[g] = qinv[g0 + g]; m[g] = kLowest; mv[g] = kLowest; l[g] = 0.f; acc[g] = 0.f; }
        bool ok = true;
        auto add_output = [&](int c) {                               // group c's product into acc
            if (kByTiles && half != 0) return;                       // (one thread a dim is enough)
            ok = ok && tc::mbar_wait_warp(bar(kBarO), c & 1, abort_flag, cta_status);
            if (!ok) return;
            tc::tc_fence_after();
            float o[8], o2[8];
            tmem_ld8(trow + set * 16, o);
            tmem_ld8(trow + set * 16 + 8, o2);
#pragma unroll
            for (int g = 0; g < kHalf; ++g) acc[g] += fmaf(fmaf(fmaf(o2[4 + g], 0.0625f, o2[g]), 0.0625f, o[4 + g]), 0.0625f, o[g]);
        };
        for (int c = 0; c < groups; ++c) {
            const int n = min(kGroup, nt - c * kGroup), first_key = key0 + c * kGroup * kTile;
            const int t0 = kByTiles ? (c * kGroup + part_of) & 1 : 0;  // this half's first tile of the group
            const float *in = info + (c % 3) * 2 * kMostPages;
            if (c + 1 < groups) scales(c + 1, next_k, next_lv);
            float top[kHalf], topv[kHalf];
#pragma unroll
            for (int g = 0; g < kHalf; ++g) { top[g] = kLowest; topv[g] = kLowest; }
            for (int t = t0; t < n; t += parts) {
                ok = ok && tc::mbar_wait_warp(bar(kBarS + (c & 1) * kGroup + t), (c >> 1) & 1, abort_flag, cta_status);
                if (!ok) continue;
                tc::tc_fence_after();
                float s[8];
                tmem_ld8(tcols + kColS + ((c & 1) * kGroup + t) * kQCols, s);
                if (first_key + t * kTile + row < r.rows) {
                    const int j = (t * kTile + row) >> A.page_shift;
                    const float ks = in[j], lv = in[kMostPages + j];
#pragma unroll
                    for (int g = 0; g < kHalf; ++g) {
                        const float z = fmaf(s[4 + g], 0.0625f, s[g]) * (ks * cq[g]);
                        top[g] = fmaxf(top[g], z);
                        topv[g] = fmaxf(topv[g], z + lv);
                    }
                }
            }
            float *all = red + (c & 1) * 8 * 2 * kHalf;
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    top[g] = fmaxf(top[g], __shfl_xor_sync(0xFFFFFFFFu, top[g], o));
                    topv[g] = fmaxf(topv[g], __shfl_xor_sync(0xFFFFFFFFu, topv[g], o));
                }
                if (lane == 0) { all[(e >> 5) * 2 * kHalf + g] = top[g]; all[(e >> 5) * 2 * kHalf + kHalf + g] = topv[g]; }
            }
            // (three buffers: a slower thread may still read the scales of the group before, and nobody those before it)
            if (c + 1 < groups && e < kMostPages) {
                float *to = info + ((c + 1) % 3) * 2 * kMostPages;
                to[e] = next_k; to[kMostPages + e] = next_lv;
            }
            if (c > 0) {                                             // (before the barrier: behind it this group's product may begin)
                add_output(c - 1);
                tc::tc_fence_before();
            }
            epi_sync();
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                float a = m[g], b = mv[g];
#pragma unroll
                for (int w = 0; w < 4 * parts; ++w) {
                    const float *of = all + (4 * (kByTiles ? 0 : half) + w) * 2 * kHalf;
                    a = fmaxf(a, of[g]);
                    b = fmaxf(b, of[kHalf + g]);
                }
                l[g] *= tc::ex2(m[g] - a);
                acc[g] *= tc::ex2(mv[g] - b);
                m[g] = a; mv[g] = b;
            }
            for (int t = t0; t < n; t += parts) {
                const int i = c * kGroup + t, pb = i & 1;
                ok = ok && tc::mbar_wait_warp(bar(kBarPEmpty + pb), ((i >> 1) & 1) ^ 1, abort_flag, cta_status);
                if (!ok) continue;
                float s[8];
                tmem_ld8(tcols + kColS + ((c & 1) * kGroup + t) * kQCols, s);
                const bool valid = first_key + t * kTile + row < r.rows;
                const int j = (t * kTile + row) >> A.page_shift;
                const float ks = in[j], lv = in[kMostPages + j] + 8.f;                  // (weights times 256)
                // rows of the operand by half, piece, head: their number's last three bits, which the swizzle takes, are those of 4 piece + head
                const uint32_t at = base + kSmemP + pb * kPCols * 128 + set * 16 * 128 + (row & 15);
#pragma unroll
                for (int g = 0; g < kHalf; g += 2) {
                    if (g0 + g < G) {
                        float w[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float z = fmaf(s[4 + g + k], 0.0625f, s[g + k]) * (ks * cq[g + k]);
                            l[g + k] += valid ? tc::ex2(z - m[g + k]) : 0.f;
                            w[k] = valid ? tc::ex2(z + lv - mv[g + k]) : 0.f;
                        }
                        uint32_t piece[4];
                        four_pieces(w[0], w[1], piece);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int n0 = 4 * k + g, n1 = n0 + 1;
                            sts8(at + n0 * 128 + (((row >> 4) ^ (n0 & 7)) << 4), piece[k]);
                            sts8(at + n1 * 128 + (((row >> 4) ^ (n1 & 7)) << 4), piece[k] >> 8);
                        }
                    }
                }
                if (i == nt - 1 && first_key + (t + 1) * kTile > r.rows) {
                    // Rows of V behind the unit's last one: zeros, since a weight of zero times a NaN would not be nothing.  The range's last
                    // tile is the last one the loader sends; the stage's load before it has been waited for (it is a K tile of this group, or a V tile
                    // whose product is done: of the group before, or four and more tiles back in this one).
                    const int load = 2 * nt - 1, at_stage = load % kStages;
                    ok = ok && tc::mbar_wait_warp(bar(kBarFull + at_stage), (load / kStages) & 1, abort_flag, cta_status);
                    if (!ok) continue;
                    if (!valid)
                        for (int k = half * (2 - parts) * 4; k < (kByTiles ? 8 : half * 4 + 4); ++k)
                            tc::sts128(base + at_stage * kStageBytes + row * 128 + k * 16, 0.f, 0.f, 0.f, 0.f);
                }
                fence_proxy_async();
                tc::tc_fence_before();
                tc::mbar_arrive(bar(kBarPFull + pb));
            }
        }
        add_output(groups - 1);
        float *sums = red + (groups & 1) * 8 * 2 * kHalf;              // (not what the last group's maxima are read from)
#pragma unroll
        for (int g = 0; g < kHalf; ++g) {
            l[g] = warp_sum(l[g]);
            if (lane == 0) sums[(e >> 5) * 2 * kHalf + g] = l[g];
        }
        epi_sync();
        float *out = A.out + ((int64_t)r.u * A.Hq + r.h * G) * 128 + row, *part = A.part + (int64_t)blockIdx.x * record;
        if (!kByTiles || half == 0) {
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                if (g0 + g < G && ok) {
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < 4 * parts; ++w) sum += sums[(4 * (kByTiles ? 0 : half) + w) * 2 * kHalf + g];
                    const float o = acc[g] * tc::ex2(mv[g] - m[g] - 8.f);       // relative to the logits' maximum
                    if (r.n_split == 1) {
                        out[(g0 + g) * 128] = o / sum;
                    } else {
                        part[(g0 + g) * 128 + row] = o;
                        if (row == 0) { part[G * 128 + g0 + g] = m[g]; part[G * 128 + G + g0 + g] = sum; }
                    }
                }
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 1) tc::tmem_dealloc(tmem, kTmemCols);
    if (threadIdx.x == 0 && *abort_flag != 0) report(A.status, *cta_status);
    if (!work || r.n_split == 1) return;
    if (threadIdx.x == 32) *last = take_ticket(ticket, seen, A.call, r.n_split);
    __syncthreads();
    if (!*last) return;
    join_ranges<kThreads, 128>(A.part + ((int64_t)blockIdx.x - (int64_t)r.split * A.Hkv) * record, (int64_t)A.Hkv * record, r.n_split, G,
                               A.out + ((int64_t)r.u * A.Hq + r.h * G) * 128);
}

}  // namespace ptc
}  // namespace paged
}  // namespace flowmm
