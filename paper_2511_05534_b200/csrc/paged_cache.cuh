// The paged 8-bit cache: block tables and slot maps from request lengths, rows quantised into pages, pages read back.
//
// Layout: a pool of pages [n_pages, Hkv, page_size, D] of e4m3 codes for K and one for V, each with one scale per page and
// KV head.  A page's value is code * scale.  The scale is a power of two, 2^ceil(log2(largest / 448)): e4m3 is a floating
// format, so a power of two costs no bit of the codes, at most a binade of their range, and a page whose scale grows because
// a larger row is appended has its older codes rescaled exactly (but for codes that become subnormal).
#pragma once
#include "common.cuh"

namespace flowmm {
namespace paged {

constexpr int kStatusPool = 11;             // FLOWMM_ERR_POOL
constexpr int kLowestExponent = -96;        // of a scale: of pages without anything, and of anything smaller than 448 * 2^-96

__device__ __forceinline__ void report(int *status, int code) { atomicCAS(status, 0, code); }

// ---- e4m3 ----------------------------------------------------------------------------------------
// two fp32 to two e4m3 codes (round to nearest even; NaN stays NaN; at most 448 in size by the callers' scales)
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    unsigned short c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
    return c;
}
// two e4m3 codes to two fp32 (exact, by way of fp16)
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)codes));
    float2 f;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
__device__ __forceinline__ void from_e4m3x16(const uint4 &c, float (&x)[16]) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = from_e4m3x2(w[i]), b = from_e4m3x2(w[i] >> 16);
        x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = b.x; x[4 * i + 3] = b.y;
    }
}
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Exponent of the smallest power of two s with size <= 448 s (448 = 1.75 * 2^8), size finite and not negative.
__device__ __forceinline__ int scale_exponent(float size) {
    const uint32_t b = __float_as_uint(size);
    return max(kLowestExponent, (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}
// The smallest such exponent that a page's scale does not exceed (a scale that no store has written may be anything).
__device__ __forceinline__ int held_exponent(float scale) {
    if (!(scale > 0.f)) return kLowestExponent;
    const uint32_t b = __float_as_uint(scale);
    return min(120, max(kLowestExponent, (int)(b >> 23) - 127 + ((b & 0x7FFFFFu) != 0u ? 1 : 0)));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// ---- block tables and slot maps ------------------------------------------------------------------
struct PlanArgs {
    const int *grow, *rows;            // [U]
    int *rows_out;                     // [U]
    int *ring;                         // [n_pages]
    const int *state;                  // {head, count}
    int *state_out;
    int *table;                        // [U, max_pages]
    int *slots;                        // [U, T] or null
    int *status;
    int U, T, page, page_shift, n_pages, max_pages, chunks;
};
constexpr int kPlanThreads = 512, kPlanChunk = 256;        // slots of a unit that a warp takes at once

// a place counted on from one inside the ring, fewer than n further (pages taken: never more than are free)
__device__ __forceinline__ unsigned ring_place(unsigned i, unsigned n) { return i >= n ? i - n : i; }

struct PlanUnit { int rows, grow, held, want; unsigned at, to; };   // grow < 0 too: rows to drop; at, to: first place in the ring to take from, to give to

// Units take pages in their order, so where a unit takes from is a prefix sum over the units before it.  Every block goes over
// all units (a load, a scan of two numbers), which costs a microsecond for 512 of them and spares a second launch or a grid-wide
// barrier; the pages and slots that follow are shared out by warps over all blocks.  Nothing is read that another block writes:
// the rows and the ring's state go to arrays of their own, table entries that are read are pages held before, and places of the
// ring that are written are not among the free ones.
__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const PlanArgs A) {
    __shared__ PlanUnit unit[kPlanThreads];
    __shared__ long long warp_need[kPlanThreads / 32], warp_back[kPlanThreads / 32];
    __shared__ unsigned taken_max;
    predecessor_done();
    successor_may_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = A.state[0], count = A.state[1];
    const bool sound = head >= 0 && head < A.n_pages && count >= 0 && count <= A.n_pages;
    const bool first = blockIdx.x == 0;
    if (tid == 0) {
        taken_max = 0;
        if (!sound && first) report(A.status, kStatusIndex);
    }
    const long long most = (long long)A.max_pages << A.page_shift;
    const unsigned n = A.n_pages;
    long long need_before = 0, back_before = 0;                    // of the units of earlier tiles
    unsigned largest = 0;                                          // page number that this thread has met
    for (int u0 = 0; u0 < A.U; u0 += kPlanThreads) {
        const int u = u0 + tid;
        PlanUnit me = {0, 0, 0, 0, 0u, 0u};
        long long need = 0, back = 0;
        bool ok = false;
        if (u < A.U) {
            me.rows = A.rows[u];
            const int grow = A.grow[u];
            const long long next = max(0ll, (long long)me.rows + grow);
            const bool valid = sound && me.rows >= 0 && me.rows <= most;
            ok = valid && next <= most && (A.slots == nullptr || grow <= A.T);
            if (!valid && first) report(A.status, kStatusIndex);
            me.held = (int)(((long long)(valid ? me.rows : 0) + A.page - 1) >> A.page_shift);
            me.want = ok ? (int)((next + A.page - 1) >> A.page_shift) : me.held;
            me.grow = grow;
            need = max(0, me.want - me.held);
            back = max(0, me.held - me.want);
        }
        long long upto = need, given = back;                       // inclusive sums
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long a = __shfl_up_sync(0xFFFFFFFFu, upto, o), b = __shfl_up_sync(0xFFFFFFFFu, given, o);
            if (lane >= o) { upto += a; given += b; }
        }
        __syncthreads();                                           // (the tile before is done with unit[] and the warps' sums)
        if (lane == 31) { warp_need[warp] = upto; warp_back[warp] = given; }
        __syncthreads();
        long long need_tile = 0, back_tile = 0;
#pragma unroll
        for (int w = 0; w < kPlanThreads / 32; ++w) {
            if (w < warp) { upto += warp_need[w]; given += warp_back[w]; }
            need_tile += warp_need[w]; back_tile += warp_back[w];
        }
        upto += need_before; given += back_before;
        if (u < A.U) {
            if (need > 0 && upto > count) ok = false;
            if (!ok) { me.want = me.held; me.grow = 0; }
            if (ok && need > 0) atomicMax(&taken_max, (unsigned)upto);
            if (ok && need > 0) me.at = ring_place(head + (unsigned)(upto - need), n);
            if (back > 0) {                                        // (a remainder only where more comes back than the ring can hold)
                const unsigned long long to = (unsigned long long)head + count + given - back;
                me.to = to < 2ull * n ? ring_place((unsigned)to, n) : (unsigned)(to % n);
            }
            if (first) {
                A.rows_out[u] = ok ? max(0, me.rows + me.grow) : me.rows;
                if (!ok) report(A.status, kStatusPool);
            }
        }
        unit[tid] = me;
        need_before += need_tile; back_before += back_tile;
        __syncthreads();
        // pages and slots: a warp takes kPlanChunk slots of a unit, and with the first of them the unit's pages
        const int here = min(kPlanThreads, A.U - u0), items = here * A.chunks;
        for (int item = blockIdx.x * (kPlanThreads / 32) + warp; item < items; item += gridDim.x * (kPlanThreads / 32)) {
            const int i = A.chunks == 1 ? item : item / A.chunks, c = item - i * A.chunks;
            const PlanUnit p = unit[i];
            int *row = A.table + (int64_t)(u0 + i) * A.max_pages;
            if (c == 0) {
                // (four reads on their way before the first write: an ended request gives hundreds of pages back)
                for (int j0 = p.held + lane; j0 < p.want; j0 += 128) {
                    int x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = j0 + 32 * k < p.want ? A.ring[ring_place(p.at + (j0 + 32 * k - p.held), n)] : 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (j0 + 32 * k < p.want) row[j0 + 32 * k] = x[k];
                        largest = max(largest, (unsigned)x[k]);
                    }
                }
                for (int j0 = p.want + lane; j0 < p.held; j0 += 128) {
                    int x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = j0 + 32 * k < p.held ? row[j0 + 32 * k] : 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        largest = max(largest, (unsigned)x[k]);
                        const unsigned to = ring_place(p.to + (j0 + 32 * k - p.want), n);
                        if (j0 + 32 * k < p.held) A.ring[to < n ? to : to % n] = x[k];      // (the remainder: more than the ring can hold)
                    }
                }
            }
            if (A.slots == nullptr) continue;
            int *out = A.slots + (int64_t)(u0 + i) * A.T;
            const int end = min(A.T, (c + 1) * kPlanChunk);
            for (int t = c * kPlanChunk + lane; t < end; t += 32) {
                int slot = -1;
                if (t < p.grow) {
                    const int pos = p.rows + t, j = pos >> A.page_shift;
                    const int id = j < p.held ? row[j] : A.ring[ring_place(p.at + (j - p.held), n)];
                    largest = max(largest, (unsigned)id);              // (the slot of a number out of range would be another page's)
                    if ((unsigned)id < n) slot = (int)(((unsigned)id << A.page_shift) | (unsigned)(pos & (A.page - 1)));
                }
                out[t] = slot;
            }
        }
    }
    if (largest >= n) report(A.status, kStatusIndex);
    if (first) {
        __syncthreads();
        if (tid == 0) {
            const long long left = (long long)count - taken_max + back_before;
            if (sound && left > A.n_pages) report(A.status, kStatusIndex);      // pages given back that were free already
            A.state_out[0] = sound ? (int)(((long long)head + taken_max) % n) : head;
            A.state_out[1] = sound ? (int)min(left, (long long)A.n_pages) : count;
        }
    }
}

// ---- rows into pages -----------------------------------------------------------------------------
struct StoreArgs {
    const void *x[2];                  // K and V rows [U, Hkv, T, D]
    const int *slots;                  // [U, T]
    uint8_t *pages[2];
    float *scale[2];
    int *status;
    int Hkv, T, page, page_shift, n_pages;
    int64_t stride[2][3];
    uint32_t items, looks;             // U * runs * Hkv * 2; U * parts of kLookRows rows, or 0
    FastDiv by_heads, by_runs, by_parts;
};

// kN codes (4 or 8) in memory as a word of that many bytes
template <int kN> struct Codes;
template <> struct Codes<4> { typedef uint32_t Word; };
template <> struct Codes<8> { typedef uint2 Word; };
__device__ __forceinline__ void unpack_codes(uint32_t c, float (&x)[4]) {
    const float2 a = from_e4m3x2(c), b = from_e4m3x2(c >> 16);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
__device__ __forceinline__ void unpack_codes(const uint2 &c, float (&x)[8]) {
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = from_e4m3x2(w[i]), b = from_e4m3x2(w[i] >> 16);
        x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = b.x; x[4 * i + 3] = b.y;
    }
}
__device__ __forceinline__ uint32_t pack_codes(const float (&x)[4]) { return to_e4m3x2(x[0], x[1]) | to_e4m3x2(x[2], x[3]) << 16; }
__device__ __forceinline__ uint2 pack_codes(const float (&x)[8]) {
    return make_uint2(to_e4m3x2(x[0], x[1]) | to_e4m3x2(x[2], x[3]) << 16, to_e4m3x2(x[4], x[5]) | to_e4m3x2(x[6], x[7]) << 16);
}

// The largest size among 16 bytes of elements, as the bits of an fp32 (bits without the sign order like the numbers; infinities and NaN are above all)
template <typename T> __device__ __forceinline__ uint32_t largest_bits(const uint4 &v);
template <> __device__ __forceinline__ uint32_t largest_bits<float>(const uint4 &v) {
    return max(max(v.x & 0x7FFFFFFFu, v.y & 0x7FFFFFFFu), max(v.z & 0x7FFFFFFFu, v.w & 0x7FFFFFFFu));
}
template <> __device__ __forceinline__ uint32_t largest_bits<__nv_bfloat16>(const uint4 &v) {
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(m << 16, m & 0xFFFF0000u);
}
constexpr uint32_t kInfinityBits = 0x7F800000u;
constexpr int kLookRows = 512;
__device__ __forceinline__ uint32_t warp_max_bits(uint32_t x) { return __reduce_max_sync(0xFFFFFFFFu, x); }

// One team of threads per (unit, page that its rows reach, KV head, K or V): the rows of the page are read once, into
// registers, their largest size found, and written as codes.  Memory bounds it: 16 bytes a thread and load, neighbours side by side, kVecs loads
// on their way at once, and nothing before them but the unit's first slot.  Next to it come the instructions for each element, so sizes are
// compared as integers, two bf16 at a time, and whether a number is finite is only asked where a thread has met one that is not
// (80 units of 1690 rows, 8 heads: 178 us with both for each element).
// Rows of a unit fill consecutive places, so the team knows from that slot which rows are its page's; every row's own
// slot is still looked at, and one that is not where it should be is left out and reported.  Rows without a place are a unit's last ones: one
// with a row behind it that has a place is found by teams of their own, kLookRows rows each, in front of the others.  (By every team, so that the pages could
// be left as they were: 72 registers for 64, 80 units of 1690 rows 132 us for 127; by the teams of one head before their rows: a call of 48 rows
// 2.85 us for 2.55.)
template <typename T, int D, int kTeam, int kVecs>
__global__ void __launch_bounds__(kTeam < 128 ? 128 : kTeam) cache_store_kernel(const StoreArgs A) {
    constexpr int kBlock = kTeam < 128 ? 128 : kTeam, kN = Elem<T>::kVec, kLanes = D / kN, kRows = kTeam / kLanes;
    typedef typename Codes<kN>::Word Word;
    __shared__ uint32_t wide[kBlock / 32];
    predecessor_done();
    successor_may_start();
    const int team = threadIdx.x / kTeam, me = threadIdx.x % kTeam, lane = me % kLanes, row0 = me / kLanes;
    const uint32_t number = blockIdx.x * (kBlock / kTeam) + team, item = number - A.looks;
    const bool looks = number < A.looks;
    bool on = !looks && item < A.items;
    const uint32_t which = item & 1u, q = item >> 1, q1 = A.by_heads.div(q), h = q - q1 * A.by_heads.d;
    const uint32_t u = A.by_runs.div(q1), run = q1 - u * A.by_runs.d;
    const int *slots = A.slots + (int64_t)(on ? u : 0) * A.T;
    const int first = on ? slots[0] : -1;
    if (first < -1 && me == 0) report(A.status, kStatusIndex);
    const int held0 = first & (A.page - 1);
    const int t0 = run == 0 ? 0 : (int)run * A.page - held0, held = run == 0 ? held0 : 0;      // the page's first new row; rows that it has already
    if (looks) {
        const uint32_t unit = A.by_parts.div(number), t0 = (number - unit * A.by_parts.d) * kLookRows;
        const int *of = A.slots + (int64_t)unit * A.T;
#pragma unroll 4
        for (int t = max(1, (int)t0) + me; t < min(A.T, (int)t0 + kLookRows); t += kTeam)
            if (of[t - 1] == -1 && of[t] != -1) report(A.status, kStatusIndex);
    }
    on = on && first >= 0 && t0 < A.T;
    const int n = on ? min(A.T - t0, A.page - held) : 0;              // rows of this page
    const T *x = static_cast<const T *>(A.x[which]) + u * A.stride[which][0] + h * A.stride[which][1] + (int64_t)t0 * A.stride[which][2] + lane * kN;
    uint4 raw[kVecs];
    int at[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = row0 + i * kRows;
        at[i] = -1;
        if (r < n) {
            raw[i] = load_raw16(x + (int64_t)r * A.stride[which][2]);
            at[i] = slots[t0 + r];
        }
    }
    const int slot = on ? slots[t0] : -1;
    const bool sound = slot < A.n_pages << A.page_shift && slot >= 0 && (slot & (A.page - 1)) == held;
    if (on && !sound && slot != -1 && me == 0) report(A.status, kStatusIndex);
    on = on && sound;
    const uint32_t page = on ? (uint32_t)slot >> A.page_shift : 0u;
    const uint32_t ph = page * A.by_heads.d + h;
    const float had = on && held > 0 ? A.scale[which][ph] : 0.f;
    uint32_t size = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = row0 + i * kRows;
        if (at[i] < 0 || !on) {
            if (at[i] != -1) report(A.status, kStatusIndex);          // (a row behind one without a place, too)
            at[i] = -1;
        } else if (at[i] != slot + r) {
            at[i] = -1;
            if (lane == 0) report(A.status, kStatusIndex);
        } else {
            size = max(size, largest_bits<T>(raw[i]));
        }
    }
    const bool odd = size >= kInfinityBits;                           // something that is not finite among this thread's
    if (odd) {
        size = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (at[i] < 0) continue;
            float f[kN];
            Elem<T>::unpack(raw[i], f);
#pragma unroll
            for (int e = 0; e < kN; ++e) size = max(size, is_finite(f[e]) ? __float_as_uint(f[e]) & 0x7FFFFFFFu : 0u);
        }
    }
    size = warp_max_bits(size);
    if (kTeam > 32) {
        if (lane_id() == 0) wide[threadIdx.x >> 5] = size;
        __syncthreads();                                              // (also: the whole team has read the page's old scale)
#pragma unroll
        for (int w = 0; w < kTeam / 32; ++w) size = max(size, wide[team * (kTeam / 32) + w]);
    } else {
        __syncwarp();
    }
    if (!on) return;
    const int e = max(held > 0 ? held_exponent(had) : kLowestExponent, scale_exponent(__uint_as_float(size)));
    const float inverse = power_of_two(-e);
    uint8_t *out = A.pages[which] + ((int64_t)ph << A.page_shift) * D + lane * kN;
    if (held > 0) {
        const float ratio = had * inverse;                            // (exact: both are powers of two)
        if (ratio != 1.f) {
            for (int r = row0; r < held; r += kRows) {
                Word *old = reinterpret_cast<Word *>(out + r * D);
                float f[kN];
                unpack_codes(*old, f);
#pragma unroll
                for (int k = 0; k < kN; ++k) f[k] *= ratio;
                *old = pack_codes(f);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        if (at[i] < 0) continue;
        float f[kN];
        Elem<T>::unpack(raw[i], f);
        if (odd) {
#pragma unroll
            for (int k = 0; k < kN; ++k) f[k] = is_finite(f[k]) ? f[k] : __uint_as_float(0x7FC00000u);
        }
#pragma unroll
        for (int k = 0; k < kN; ++k) f[k] *= inverse;
        *reinterpret_cast<Word *>(out + (held + row0 + i * kRows) * D) = pack_codes(f);
    }
    if (me == 0) A.scale[which][ph] = power_of_two(e);
}

// ---- pages into rows -----------------------------------------------------------------------------
struct LoadArgs {
    const uint8_t *pages[2];
    const float *scale[2];
    const int *table, *rows;           // [U, max_pages], [U]
    void *x[2];                        // [U, Hkv, n_rows, D]
    int *status;
    int Hkv, n_rows, page, page_shift, n_pages, max_pages;
    int64_t stride[2][3];
    FastDiv by_heads, by_chunks;
};
constexpr int kLoadThreads = 128, kLoadRows = 64;

// A block takes 64 rows of one (unit, KV head, K or V); 16 bytes of output a thread and store, neighbours side by side, all its codes on their
// way at once.  Writing bounds it.  kOnePage: pages of 64 rows and more, so that the block has one page's number and scale.
template <typename T, int D, bool kOnePage>
__global__ void __launch_bounds__(kLoadThreads) cache_load_kernel(const LoadArgs A) {
    constexpr int kN = Elem<T>::kVec, kLanes = D / kN, kRows = kLoadThreads / kLanes, kVecs = kLoadRows / kRows;
    typedef typename Codes<kN>::Word Word;
    predecessor_done();
    successor_may_start();
    const int lane = threadIdx.x % kLanes, row0 = threadIdx.x / kLanes;
    const uint32_t which = blockIdx.x & 1u, q = blockIdx.x >> 1, q1 = A.by_heads.div(q), h = q - q1 * A.by_heads.d;
    const uint32_t u = A.by_chunks.div(q1), chunk = q1 - u * A.by_chunks.d;
    const int first = (int)(chunk * kLoadRows), held = A.rows[u], most = A.max_pages << A.page_shift;
    if ((held < 0 || held > most) && threadIdx.x == 0) report(A.status, kStatusIndex);
    const int n = min(min(held, most), A.n_rows) - first;             // rows of this block
    const int *table = A.table + (int64_t)u * A.max_pages;
    if (n <= 0) return;
    constexpr int kPages = kOnePage ? 1 : kVecs;
    int id[kPages];
    Word codes[kVecs];
    float scale[kPages];
#pragma unroll
    for (int i = 0; i < kPages; ++i) {
        const int r = kOnePage ? 0 : row0 + i * kRows;
        id[i] = r < n ? table[(first + r) >> A.page_shift] : -1;
        if (r < n && (unsigned)id[i] >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); id[i] = -1; }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = row0 + i * kRows, page = id[kOnePage ? 0 : i];
        if (page < 0 || r >= n) continue;
        const int64_t ph = (int64_t)page * A.Hkv + h;
        const int at = (first + r) & (A.page - 1);
        codes[i] = *reinterpret_cast<const Word *>(A.pages[which] + ((ph << A.page_shift) + at) * D + lane * kN);
        if (!kOnePage || i == 0) scale[kOnePage ? 0 : i] = A.scale[which][ph];
    }
    T *x = static_cast<T *>(A.x[which]) + u * A.stride[which][0] + h * A.stride[which][1] + (int64_t)first * A.stride[which][2] + lane * kN;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = row0 + i * kRows;
        if (id[kOnePage ? 0 : i] < 0 || r >= n) continue;
        float f[kN];
        unpack_codes(codes[i], f);
#pragma unroll
        for (int k = 0; k < kN; ++k) f[k] *= scale[kOnePage ? 0 : i];
        Elem<T>::store16(x + (int64_t)r * A.stride[which][2], f);
    }
}

}  // namespace paged
}  // namespace flowmm
