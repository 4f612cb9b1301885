// Rotary positions: pairs of channels of queries and keys turned by an angle that goes with their token's position.
//   (a, b) -> m (a cos - b sin, b cos + a sin),   angle = position * frequency of the pair
//
// A pair's frequency is held as what a position adds to its phase, in turns, as a 64-bit fraction: position times that, modulo 2^64, is the phase,
// whole turns gone by themselves and nothing lost at far positions (an angle formed in fp32 is off by 0.03 at position 10^6).
#pragma once
#include "common.cuh"

namespace flowmm {
namespace rotary {

struct TableArgs {
    unsigned long long *phase;         // [R / 2]
    int R, scaling;                    // flowmm_rotary_scaling
    double base, factor, low, high, trained;
};

__global__ void rotary_table_kernel(const TableArgs A) {
    predecessor_done();
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= A.R / 2) return;
    constexpr double kTurn = 6.283185307179586476925;
    double f = pow(A.base, -2.0 * i / A.R);
    if (A.scaling == 1) {
        f /= A.factor;
    } else if (A.scaling == 2) {
        const double kept = fmin(1.0, fmax(0.0, (A.trained * f / kTurn - A.low) / (A.high - A.low)));
        f = kept * f + (1.0 - kept) * (f / A.factor);
    }
    const double turns = f / kTurn;
    A.phase[i] = (unsigned long long)ldexp(turns - floor(turns), 64);
}

struct Args {
    const void *x[2];                  // queries and keys [U, heads, T, D]
    void *y[2];
    const int *positions;              // [U, axes, T]
    const unsigned long long *phase;
    int heads[2];
    int each;                          // heads of a thread
    int R, axes, end0, end1;           // the first pairs that go by the second and the third position
    float amplitude;
    uint32_t rows;                     // U * T
    int64_t in[2][3], out[2][3];
    FastDiv by_rows;                   // by T
    int adjoint;
};
constexpr int kThreads = 256;

// cos and sin of a phase, a 32-bit fraction of a turn: the nearest quarter apart, what is left (an eighth at most) to fp32, where it has 25 bits and more
__device__ __forceinline__ void turn(uint32_t phase, float &c, float &s) {
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float rest = (float)(int)(phase - (quarter << 30)) * 4.656612873077393e-10f;      // of half a turn: 2^-31
    float c0, s0;
    sincospif(rest, &s0, &c0);
    c = quarter & 1u ? s0 : c0;
    s = quarter & 1u ? c0 : s0;
    if (quarter == 1u || quarter == 2u) c = -c;
    if (quarter & 2u) s = -s;
}

// A thread has two vectors of a row, so kN pairs: channels i and i + R / 2, or neighbours; the angles once for `each` heads.
template <typename T, int D, bool kPairs>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const Args A) {
    constexpr int kN = Elem<T>::kVec, kLanes = D / (2 * kN), kRows = kThreads / kLanes;
    predecessor_done();
    successor_may_start();
    const int lane = threadIdx.x % kLanes, pair = lane * kN, half = A.R / 2;
    const uint32_t row = blockIdx.x * kRows + threadIdx.x / kLanes;
    if (row >= A.rows) return;
    const uint32_t u = A.by_rows.div(row), t = row - u * A.by_rows.d;
    const bool turns = pair < half;
    const int first = kPairs || !turns ? 2 * pair : pair, second = kPairs || !turns ? first + kN : pair + half;
    float c[kN], s[kN];
    if (turns) {
        int pos[3];
#pragma unroll
        for (int a = 0; a < 3; ++a) pos[a] = a < A.axes ? A.positions[((int64_t)u * A.axes + a) * A.by_rows.d + t] : 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int p = pair + i, at = p < A.end0 ? pos[0] : p < A.end1 ? pos[1] : pos[2];
            turn((uint32_t)((A.phase[p] * (unsigned long long)(long long)at) >> 32), c[i], s[i]);
            c[i] *= A.amplitude;
            s[i] *= A.adjoint ? -A.amplitude : A.amplitude;
        }
    }
    const int all = A.heads[0] + A.heads[1], g0 = blockIdx.y * A.each, g1 = min(all, g0 + A.each);
    for (int g = g0; g < g1; ++g) {
        const int which = g >= A.heads[0], h = g - (which ? A.heads[0] : 0);
        const T *x = static_cast<const T *>(A.x[which]) + u * A.in[which][0] + h * A.in[which][1] + t * A.in[which][2];
        T *y = static_cast<T *>(A.y[which]) + u * A.out[which][0] + h * A.out[which][1] + t * A.out[which][2];
        float a[kN], b[kN];
        Elem<T>::load16(x + first, a);
        Elem<T>::load16(x + second, b);
        if (turns) {
            float p[kN], q[kN];
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
        } else {
            Elem<T>::store16(y + first, a);
            Elem<T>::store16(y + second, b);
        }
    }
}

}  // namespace rotary
}  // namespace flowmm
