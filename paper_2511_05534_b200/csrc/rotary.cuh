// Rotary positions: pairs of channels of queries and keys turned by an angle that goes with their token's position.
//   (a, b) -> m (a cos - b sin, b cos + a sin),   angle = position * frequency of the pair
//
// A pair's frequency is held as what a position adds to its phase, in turns, as a 64-bit fraction: position times that, modulo 2^64, is the phase,
// whole turns gone by themselves (an angle formed in fp32 is off by 0.03 at position 10^6).  The fraction is within 2^-63 of the true one (factors of one and more), so
// any 32-bit position has its phase, 32 bits of it, within 2^-31 turns.
#pragma once
#include <cfloat>
#include <cmath>

#include "common.cuh"
#include "flowmm.h"

namespace flowmm {
namespace rotary {

constexpr int kMostPairs = 64;         // heads of 128
struct TableArgs {
    unsigned long long *to;            // [pairs]
    unsigned long long phase[kMostPairs];
    int pairs;
};

// The fractions, on the host: a double has 53 bits, 2^-56 of a turn, which position 2^31 makes 2^-25; numbers of 64 significant bits have what is asked for.  (A factor
// below one makes more turns, and the fraction's last bits go by that.)
static_assert(LDBL_MANT_DIG >= 64, "64 significant bits");
inline unsigned long long phase_of(int i, int R, int scaling, double base, double factor, double low, double high, int trained) {
    constexpr long double kTurn = 6.283185307179586476925286766559005768394L;
    long double f = powl(base, -2.0L * i / R);
    if (scaling == FLOWMM_ROTARY_LINEAR) {
        f /= factor;
    } else if (scaling == FLOWMM_ROTARY_BY_PARTS) {
        const long double kept = fminl(1.0L, fmaxl(0.0L, (trained * f / kTurn - low) / ((long double)high - low)));
        f = kept * f + (1.0L - kept) * (f / factor);
    }
    const long double turns = f / kTurn, fraction = rintl(ldexpl(turns - floorl(turns), 64));
    return fraction < 18446744073709551616.0L ? (unsigned long long)fraction : 0ull;
}

__global__ void rotary_table_kernel(const TableArgs A) {
    predecessor_done();
    if ((int)threadIdx.x < A.pairs) A.to[threadIdx.x] = A.phase[threadIdx.x];
}

struct Args {
    const void *x[2];                  // queries and keys [U, heads, T, D]
    void *y[2];
    const int *positions;              // [U, axes, T]
    const unsigned long long *phase;
    int heads[2];
    int each;                          // heads of a block
    int R, axes, end0, end1;           // the first pairs that go by the second and the third position
    float amplitude, sine;             // of cos, of sin: turned for the adjoint
    uint32_t rows;                     // U * T
    int64_t in[2][3], out[2][3];
    FastDiv by_rows;                   // by T
};
constexpr int kThreads = 256, kFewRows = 4, kManyBytes = 4096;

// cos and sin of a phase, a 32-bit fraction of a turn: the nearest quarter apart; of what is left, an eighth of a turn at most, their Taylor series to the tenth and
// ninth power, which leave 2^-32 and 2^-29 of it.
__device__ __forceinline__ float2 turn(uint32_t phase) {
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = (float)(int)(phase - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi 2^-32
    const float y = x * x;
    float s = fmaf(y, 1.f / 362880.f, -1.f / 5040.f), c = fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
    s = fmaf(y, s, 1.f / 120.f); c = fmaf(y, c, -1.f / 720.f);
    s = fmaf(y, s, -1.f / 6.f); c = fmaf(y, c, 1.f / 24.f);
    c = fmaf(y, c, -0.5f);
    s = fmaf(y * s, x, x); c = fmaf(y, c, 1.f);
    const float2 r = quarter & 1u ? make_float2(s, c) : make_float2(c, s);
    return make_float2(quarter == 1u || quarter == 2u ? -r.x : r.x, quarter & 2u ? -r.y : r.y);
}

// A block takes four rows, or where that leaves blocks enough so many as make 4 KB of a head on end, of all or `each` heads: the angles once for all of
// them, a pair and row a thread, then a thread two vectors of a row, so kN pairs (channels i and i + R / 2, or neighbours), of every kHeads-th
// head.  Memory bounds it: each element is read and written once, 16 bytes at a time.  (33 792 rows, 72 heads of 128, 195 us for 193 of memory; with
// 1 KB on end 209, 2 KB 207; two heads on their way at once, by more registers a thread, 204; with 4 KB fp32 rows 61.6 for 61.0, with 8 KB 65.)
template <typename T, int D, bool kPairs, int kRows>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const Args A) {
    constexpr int kN = Elem<T>::kVec, kLanes = D / (2 * kN), kHeads = kThreads / (kLanes * kRows);
    __shared__ float cosine[kRows][D / 2], sine[kRows][D / 2];
    predecessor_done();
    successor_may_start();
    const uint32_t base = blockIdx.x * kRows;
    const int half = A.R / 2;
#pragma unroll
    for (int i = 0; i < (kRows * D / 2 + kThreads - 1) / kThreads; ++i) {
        const int p = (threadIdx.x + i * kThreads) % (D / 2), r = (threadIdx.x + i * kThreads) / (D / 2);
        const uint32_t row = base + r;
        if (r < kRows && p < half && row < A.rows) {
            const uint32_t u = A.by_rows.div(row), t = row - u * A.by_rows.d;
            const int axis = p < A.end0 ? 0 : p < A.end1 ? 1 : 2;
            const int at = A.positions[((int64_t)u * A.axes + axis) * A.by_rows.d + t];
            const float2 v = turn((uint32_t)((A.phase[p] * (unsigned long long)(long long)at) >> 32));
            cosine[r][p] = v.x * A.amplitude;
            sine[r][p] = v.y * A.sine;
        }
    }
    __syncthreads();
    const int lane = threadIdx.x % kLanes, r = threadIdx.x / kLanes % kRows, pair = lane * kN;
    const uint32_t row = base + r;
    if (row >= A.rows) return;
    const uint32_t u = A.by_rows.div(row), t = row - u * A.by_rows.d;
    const bool turns = pair < half;
    const int first = kPairs || !turns ? 2 * pair : pair, second = kPairs || !turns ? first + kN : pair + half;
    float c[kN], s[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        c[i] = turns ? cosine[r][pair + i] : 1.f;
        s[i] = turns ? sine[r][pair + i] : 0.f;
    }
    const int all = A.heads[0] + A.heads[1], end = min(all, ((int)blockIdx.y + 1) * A.each);
#pragma unroll 1
    for (int g = blockIdx.y * A.each + threadIdx.x / (kLanes * kRows); g < end; g += kHeads) {
        const int which = g >= A.heads[0], h = g - (which ? A.heads[0] : 0);
        const T *x = static_cast<const T *>(A.x[which]) + u * A.in[which][0] + h * A.in[which][1] + t * A.in[which][2];
        T *y = static_cast<T *>(A.y[which]) + u * A.out[which][0] + h * A.out[which][1] + t * A.out[which][2];
        const uint4 raw[2] = {load_raw16(x + first), load_raw16(x + second)};
        if (!turns) {                                                 // (as it is: not a product with one, which a NaN's bits need not survive)
            *reinterpret_cast<uint4 *>(y + first) = raw[0];
            *reinterpret_cast<uint4 *>(y + second) = raw[1];
            continue;
        }
        float a[kN], b[kN], p[kN], q[kN];
        Elem<T>::unpack(raw[0], a);
        Elem<T>::unpack(raw[1], b);
        if (kPairs) {
#pragma unroll
            for (int i = 0; i < kN; i += 2) {
                p[i] = a[i] * c[i / 2] - a[i + 1] * s[i / 2];
                p[i + 1] = a[i + 1] * c[i / 2] + a[i] * s[i / 2];
                q[i] = b[i] * c[kN / 2 + i / 2] - b[i + 1] * s[kN / 2 + i / 2];
                q[i + 1] = b[i + 1] * c[kN / 2 + i / 2] + b[i] * s[kN / 2 + i / 2];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) { p[i] = a[i] * c[i] - b[i] * s[i]; q[i] = b[i] * c[i] + a[i] * s[i]; }
        }
        Elem<T>::store16(y + first, p);
        Elem<T>::store16(y + second, q);
    }
}

}  // namespace rotary
}  // namespace flowmm
