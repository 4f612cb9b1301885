// The paged 4-bit cache: rows quantised into pages, pages read back.
//
// Layout: pages of codes [n_pages, Hkv, page_size, D / 2], two channels a byte (the even one in the low half), and of scales
// [n_pages, Hkv, page_size, D / 16], one for 16 neighbouring channels of a row.  A code is e2m1 (sign, two exponent bits, one of mantissa: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6), a scale the upper byte of a positive fp16 without its lowest seven bits (five exponent bits, three of mantissa),
// so widening it is a shift, its range needs no second scale, and the product of the two is an fp16 exactly.  Rows do not depend on one
// another: a row that is appended changes nothing else, and any row may go anywhere.
// (Random keys with a few strong channels, the attention's output against the one without quantising, root mean square relative to its own:
// so 0.159; integers with a scale of 16 bits for 32 channels, as many bits, 0.219; integers with a scale and an offset for 32, 5 bits, 0.155;
// e2m1 with a power of two for 32, 4.25 bits, 0.277; scales rounded up and not to the nearest 0.184.)
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"
#include "tc_common.cuh"

namespace flowmm {
namespace nibble {

using paged::report;

constexpr int kGroup = 16;                       // channels with a scale
constexpr uint32_t kLeastScale = 0x38800000u;    // 2^-14, fp16's least normal number, as the bits of an fp32
constexpr uint32_t kMostScale = 0x46200000u;     // 10240: the largest scale whose products with codes (6 at most) are fp16 numbers
constexpr uint32_t kScaleBias = 896u;            // bits >> 20 of the fp32 minus the byte: 8 (127 - 15)
constexpr uint32_t kNanScale = 255u;

// The scale of a group whose largest size has these bits (finite): a sixth of it rounded to four significant bits, to the nearest, ties to even.
// `low` is a sixth cut off, or, where the product was rounded onto the next number, that: what lies half way to the one above it is compared exactly,
// as six times that has eight bits at most.
__device__ __forceinline__ uint32_t scale_bits(uint32_t size) {
    const uint32_t low = __float_as_uint(__uint_as_float(size) * (1.f / 6.f)) & 0xFFF00000u;
    const uint32_t half = __float_as_uint(6.f * __uint_as_float(low + 0x00080000u));
    const uint32_t b = size > half - (low >> 20 & 1u) ? low + 0x00100000u : low;      // (positive numbers are ordered as their bits are)
    return min(max(b, kLeastScale), kMostScale);
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Eight quotients x / s as codes, all signs turned (to be turned back with 0x88888888).  Borders between codes are hit exactly - they have three bits, s has
// four - and what is next to a border must not be taken onto it, so a product with the reciprocal (within 2^-22) is corrected once by its exact
// remainder: then it is within 2^-44 of the quotient before its rounding, and a quotient next to a border is 0.53 of a step or more away from it, as
// s's significand is 15 / 8 at most.  (Two at a time; signs turned because x - s y keeps the sign of zeros then.)
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float s, float inverse) {
    const float2 step = make_float2(s, s), minus = make_float2(-inverse, -inverse);
    float2 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = make_float2(x[2 * i], x[2 * i + 1]), y0 = tc::fmul2(v, minus);
        y[i] = tc::ffma2(tc::ffma2(y0, step, v), minus, y0);
    }
    uint32_t c;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(c)
        : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
    return c;
}
// Eight codes as four pairs of fp16, neighbouring channels together.
__device__ __forceinline__ void widen8(uint32_t c, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(c));
}
__device__ __forceinline__ float2 from_half2(uint32_t h) {
    float2 f;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return from_half2(byte << 7).x; }
__device__ __forceinline__ void values8(uint32_t codes, uint32_t scale, float (&x)[8]) {
    uint32_t h[4];
    widen8(codes, h);
    const float s = scale_value(scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = from_half2(h[i]);
        x[2 * i] = f.x * s;
        x[2 * i + 1] = f.y * s;
    }
}

// eight neighbouring elements as they are in memory
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = load_raw16(p); }
    __device__ __forceinline__ uint32_t size() const { return paged::largest_bits<__nv_bfloat16>(v); }
    __device__ __forceinline__ void get(float (&x)[8]) const { Elem<__nv_bfloat16>::unpack(v, x); }
};
template <> struct Eight<float> {
    uint4 v[2];
    __device__ __forceinline__ void load(const float *p) { v[0] = load_raw16(p); v[1] = load_raw16(p + 4); }
    __device__ __forceinline__ uint32_t size() const { return max(paged::largest_bits<float>(v[0]), paged::largest_bits<float>(v[1])); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    }
};

constexpr int kCopyThreads = 256;

// ---- rows into pages -----------------------------------------------------------------------------
struct StoreArgs {
    const void *x[2];                  // K and V rows [U, Hkv, T, D]
    const int *slots;                  // [U, T]
    uint8_t *pages[2], *scale[2];
    int *status;
    int T, Hkv, page_shift, n_pages;
    uint32_t rows;                     // of few: U * Hkv * T
    int64_t stride[2][3];
    FastDiv by_heads, by_rows;         // by Hkv; by T, or by the parts that a unit's rows make
};

// A thread has a group, 16 channels of a row, and kVecs rows on their way at once.  kFew: calls of few rows a unit; rows stand in a line, by unit, KV head and
// row.  Else a block takes kRows * kVecs rows of one unit and head, so that what addresses need is found once.  Memory bounds it as long as a
// group takes no more than about 200 instructions: so sizes are compared as integers, two bf16 at a time, and quotients are formed in pairs.
// 80 units of 1690 rows, 8 heads of 128: 105 us, 110 of memory (part of what is written stays in L2); with eight channels a thread, divisions and
// addresses for each of them 211.  fp32, 40 units: 91 us, 98 of memory.  One row of 4 units: 1.6 us.
template <typename T, int D, int kVecs, bool kFew>
__global__ void __launch_bounds__(kCopyThreads) nibble_store_kernel(const StoreArgs A) {
    constexpr int kLanes = D / kGroup, kRows = kCopyThreads / kLanes;
    predecessor_done();
    successor_may_start();
    const int lane = threadIdx.x % kLanes, row0 = threadIdx.x / kLanes;
    const uint32_t which = blockIdx.y;
    uint32_t u = 0, h = 0, first = blockIdx.x * (kRows * kVecs), end = A.rows;
    if (!kFew) {
        const uint32_t uh = A.by_rows.div(blockIdx.x);
        first = (blockIdx.x - uh * A.by_rows.d) * (kRows * kVecs);
        end = A.T;
        u = A.by_heads.div(uh);
        h = uh - u * A.by_heads.d;
    }
    const int *slots = A.slots + (int64_t)u * A.T;
    const T *x = static_cast<const T *>(A.x[which]) + u * A.stride[which][0] + h * A.stride[which][1] + lane * kGroup;
    Eight<T> raw[kVecs][2];
    int slot[kVecs];
    uint32_t head[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const uint32_t r = first + row0 + i * kRows;
        slot[i] = -1;
        head[i] = h;
        if (r >= end) continue;
        const T *from = x;
        if (kFew) {
            const uint32_t uh = A.by_rows.div(r), t = r - uh * A.by_rows.d, unit = A.by_heads.div(uh);
            head[i] = uh - unit * A.by_heads.d;
            slot[i] = slots[(int64_t)unit * A.T + t];
            from += unit * A.stride[which][0] + head[i] * A.stride[which][1] + t * A.stride[which][2];
        } else {
            slot[i] = slots[r];
            from += r * A.stride[which][2];
        }
        raw[i][0].load(from);
        raw[i][1].load(from + 8);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        if (slot[i] < 0 || slot[i] >= A.n_pages << A.page_shift) {
            if (slot[i] != -1) report(A.status, kStatusIndex);
            continue;
        }
        const uint32_t size = max(raw[i][0].size(), raw[i][1].size());
        const int64_t at = ((int64_t)((uint64_t)((uint32_t)slot[i] >> A.page_shift) * ((uint32_t)A.Hkv << A.page_shift))) +
                           ((head[i] << A.page_shift) + ((uint32_t)slot[i] & ((1u << A.page_shift) - 1u)));
        const uint32_t b = scale_bits(size);
        const float s = __uint_as_float(b), inverse = reciprocal(s);
        float f[8];
        uint2 codes;
        raw[i][0].get(f);
        codes.x = codes8(f, s, inverse) ^ 0x88888888u;
        raw[i][1].get(f);
        codes.y = codes8(f, s, inverse) ^ 0x88888888u;
        uint32_t byte = (b >> 20) - kScaleBias;
        if (size >= paged::kInfinityBits) { codes = make_uint2(0u, 0u); byte = kNanScale; }
        *reinterpret_cast<uint2 *>(A.pages[which] + at * (D / 2) + lane * 8) = codes;
        A.scale[which][at * (D / kGroup) + lane] = (uint8_t)byte;
    }
}

// ---- pages into rows -----------------------------------------------------------------------------
struct LoadArgs {
    const uint8_t *pages[2], *scale[2];
    const int *table, *rows;           // [U, max_pages], [U]
    void *x[2];                        // [U, Hkv, n_rows, D]
    int *status;
    int n_rows, page_shift, n_pages, max_pages;
    int64_t stride[2][3];
    FastDiv by_heads, by_chunks;
};
constexpr int kLoadRows = 64, kLoadThreads = 128;

// The codes of 16 bytes of output, and what they stand for.
template <typename T> struct Codes;
template <> struct Codes<__nv_bfloat16> {
    typedef uint32_t Word;
    static __device__ __forceinline__ void store(__nv_bfloat16 *to, Word c, uint32_t scale) {
        float x[8];
        values8(c, scale, x);
        Elem<__nv_bfloat16>::store16(to, x);
    }
};
template <> struct Codes<float> {
    typedef unsigned short Word;
    static __device__ __forceinline__ void store(float *to, Word c, uint32_t scale) {
        uint32_t h[2];
        asm("{\n\t.reg .b8 a, b;\n\tmov.b16 {a, b}, %2;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t}" : "=r"(h[0]), "=r"(h[1]) : "h"(c));
        const float2 a = from_half2(h[0]), b = from_half2(h[1]);
        const float s = scale_value(scale);
        *reinterpret_cast<float4 *>(to) = make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
    }
};

// A block takes 64 rows of one (unit, KV head, K or V); a thread has 16 bytes of output of every kRows-th row, neighbours side by side, eight rows' codes
// and scales on their way at once.  Writing bounds it, next to it the instructions for each 16 bytes, so that addresses are formed once where all
// rows are on one page (kOnePage: pages of 64 rows and more).  80 units of up to 1690 rows, 8 heads of 128: 70 us, 65 of memory (addresses for each
// 16 bytes: 92); pages of 16 rows 70; fp32, 40 units 62 us, 57 of memory; 28 units of up to 640 rows, 4 heads, 6.4 us, 4.2 of memory.
template <typename T, int D, bool kOnePage>
__global__ void __launch_bounds__(kLoadThreads) nibble_load_kernel(const LoadArgs A) {
    constexpr int kN = Elem<T>::kVec, kLanes = D / kN, kRows = kLoadThreads / kLanes, kVecs = kLoadRows / kRows < 8 ? kLoadRows / kRows : 8;
    typedef typename Codes<T>::Word Word;
    predecessor_done();
    successor_may_start();
    const int lane = threadIdx.x % kLanes, row0 = threadIdx.x / kLanes, page = 1 << A.page_shift;
    const uint32_t which = blockIdx.x & 1u, q = blockIdx.x >> 1, q1 = A.by_heads.div(q), h = q - q1 * A.by_heads.d;
    const uint32_t u = A.by_chunks.div(q1), chunk = q1 - u * A.by_chunks.d;
    const int first = (int)(chunk * kLoadRows), held = A.rows[u], most = A.max_pages << A.page_shift;
    const int *table = A.table + (int64_t)u * A.max_pages + (first >> A.page_shift);
    if ((held < 0 || held > most) && threadIdx.x == 0) report(A.status, kStatusIndex);
    const int n = min(kLoadRows, min(min(held, most), A.n_rows) - first);             // rows of this block
    if (n <= 0) return;
    const uint8_t *codes = A.pages[which] + lane * kN / 2, *scales = A.scale[which] + lane * kN / kGroup;
    const uint32_t page_rows = A.by_heads.d << A.page_shift;
    if (kOnePage) {
        int id = table[0];
        if ((unsigned)id >= (unsigned)A.n_pages) { if (threadIdx.x == 0) report(A.status, kStatusIndex); return; }
        const int64_t row = (int64_t)((uint64_t)(uint32_t)id * page_rows) + ((h << A.page_shift) + (first & (page - 1)) + row0);
        codes += row * (D / 2);
        scales += row * (D / kGroup);
    }
    T *x = static_cast<T *>(A.x[which]) + u * A.stride[which][0] + h * A.stride[which][1] + (int64_t)(first + row0) * A.stride[which][2] + lane * kN;
    const int64_t step = kRows * A.stride[which][2];
#pragma unroll 1
    for (int r0 = 0; r0 < n; r0 += kVecs * kRows) {
        Word c[kVecs];
        uint8_t s[kVecs];
        if (kOnePage && r0 + kVecs * kRows <= n) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                c[i] = *reinterpret_cast<const Word *>(codes + (r0 + i * kRows) * (D / 2));
                s[i] = scales[(r0 + i * kRows) * (D / kGroup)];
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                Codes<T>::store(x, c[i], s[i]);
                x += step;
            }
            continue;
        }
        int id[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int r = row0 + r0 + i * kRows;
            id[i] = r < n ? (kOnePage ? 0 : table[r >> A.page_shift]) : -1;            // (first is the first row of a page)
            if (r < n && (unsigned)id[i] >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); id[i] = -1; }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (id[i] < 0) continue;
            const int64_t row = kOnePage ? r0 + i * kRows
                                         : (int64_t)((uint64_t)(uint32_t)id[i] * page_rows) + ((h << A.page_shift) + ((row0 + r0 + i * kRows) & (page - 1)));
            c[i] = *reinterpret_cast<const Word *>(codes + row * (D / 2));
            s[i] = scales[row * (D / kGroup)];
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (id[i] >= 0) Codes<T>::store(x, c[i], s[i]);
            x += step;
        }
    }
}

}  // namespace nibble
}  // namespace flowmm
