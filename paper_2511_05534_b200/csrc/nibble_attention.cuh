// Decode attention over the paged 4-bit cache: one new query per query head, lengths of their own for every unit.
//   o = sum_j softmax_j(scale * q . k_j) v_j,   k_j, v_j: rows of e2m1 codes times their groups' scales
//
// One pass over K and V with a running maximum and sum.  A row of 128 channels is 72 bytes of K and 72 of V for 4 G 128 flops: memory has one for an SM every
// 6.3 clocks.  The products go to the tensor cores, the codes are widened in registers, by warps that feed their own matrix instructions (mma.sync, fp16
// operands, fp32 sums): a code times its scale is an fp16 number exactly, one conversion and one packed product for two of them.
// (tcgen05 takes its operands from shared or tensor memory: 256 bytes a row written and read there for the 72 that came, 4 clocks of the 6.3; and e2m1 operands
// with scales of their own, which it takes as they are, would want queries and weights in 4 or 8 bits.)
//   S[key, head] = K Q^T:  16 keys on the wide side, eight query heads, the most there are, on the narrow one
//   O^T[channel, head] = V^T W^T:  16 channels on the wide side; the weights go from the first product's layout to the second's by a transpose in registers
// Which channel and which key stand at which place of an operand is free as long as both operands agree: a lane takes 16 neighbouring bytes of a K row and
// 8 of a V row, one scale for all channels that it has of a V row, and ends with 16 neighbouring channels of two query heads.
// bf16: a query is an fp16 number times a power of two exactly, a weight is rounded to fp16 (2^-11, where the output is rounded to 2^-8: one element in 70 to 700 becomes
// its neighbour by that; the sum that divides takes weights unrounded, as it has them in fp32); fp32: both are the sum of two fp16 numbers, each product is two.  The largest weight is 2^10 to 2^15 (fp32: 2^14), so that fp16 holds others to full precision down to 2^-24 of
// it, and two of them to 2^-21 of themselves down to 2^-18 of it, both to 2^-35 (fp32: 2^-39) of it below.
//
// A warp works by itself: tiles of 64 rows come into its own ring of three half tiles (K and V in turn), 16 bytes a lane and copy, two ahead; it keeps the
// maximum, the sum and the output of the head that it is at.  Twelve warps are on an SM, as many as 168 registers and 18 KB of shared memory each allow.
// (32 rows a tile and sixteen warps of 128 registers spilled: 101 us where this took 84; ten warps 94; a tile's V together with the next one's K, in a ring of four,
// 85 where this took 79; loops over the 16 keys not unrolled 87.)  What it costs is instructions: 1040 for a tile of
// 128 channels, of which 860 widen and multiply, so addresses are formed from one page number for a tile where pages have 64 rows (bulk copies by one thread
// took 40 instructions each), and outputs are rescaled only where fp16 asks for it.
// Measured: 16 sequences of up to 33 792 rows, 8 heads of 8 query heads, 386 MB, 79 us, 60 of memory: 5.5 TB/s while all blocks run, 6 us from the launch to the first
// tile, and an end of 14 us in which blocks finish one after the other, since equal pieces take SMs 76 to 90 us.  64 sequences of up to 1690 rows, 74 MB, 24.8 us, 11.5
// of memory.  One sequence of 218 rows 5.0 us: lengths and table 0.6, the first tile 0.9, its products 1.2, joining the warps' records 0.9, the launch.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "nibble_cache.cuh"
#include "paged_attention.cuh"
#include "tc_common.cuh"

namespace flowmm {
namespace nibble {

struct AttnArgs {
    const void *q;                     // [U, Hq, D] dense
    const uint8_t *pages[2];           // of K and V [n_pages, Hkv, page, D / 2]
    const uint8_t *scale[2];           // [n_pages, Hkv, page, D / 16]
    const int *table, *rows;           // [U, max_pages], [U]
    void *out;                         // [U, Hq, D]
    float *part;                       // two records a block (paged::record_floats)
    int4 *cut_heads;                   // [blocks], as paged::AttnArgs has it; null: no head is cut
    int *status;
    int share;                         // Share
    int U, Hq, Hkv, G, page_shift, n_pages, max_pages;
    float scale_log2;
    FastDiv by_heads;                  // by Hkv
};

enum Share { kOneHead, kTwoHeads, kHeadsInLine, kCutHeads };          // what a block has
constexpr int kTile = 64, kWarps = 6, kBlocks = 2, kAttnThreads = kWarps * 32, kHeads = 8;      // blocks of an SM
constexpr float kLowest = paged::kLowest;
// Weights are 2^(10 + (product - reference) factor) (fp32 rows: 14): the reference is a maximum of the products q . k as they come from the matrix instructions, and set
// again only when a weight would be above 2^15.  Differences are formed before they are scaled, so the largest product's weight is 2^10 however large the logits are
// (2^(logit - reference) by one multiply-add lost it where a step of fp32 at the logit is above 10: zeros and NaN from 2^28 on).
constexpr float kMostExponent = 15.f;

// What a warp has in shared memory: three half tiles (64 rows of K or of V: codes, then scales), K and V in turn, and a record.
template <int D> struct Lay {
    static constexpr uint32_t kCodes = kTile * D / 2, kScales = kTile * D / kGroup, kHalf = kCodes + kScales;
    static constexpr uint32_t kRecord = kHeads * (D + 2) * 4;
    static constexpr uint32_t kRecords = kWarps * 3 * kHalf, kMeta = kRecords + kWarps * kRecord, kBytes = kMeta + kWarps * 32;
    static_assert(kRecord <= 3 * kHalf && kBlocks * (kBytes + 1024) <= 228 * 1024, "blocks of an SM");
};

// ---- how the work is shared out ------------------------------------------------------------------
// The tiles of all heads stand in a line, by unit, head and key.  With at most as many heads as blocks a block has a range of one head, `per` tiles or what
// remains of it (ranges no longer than kSwitchTiles above an even share); else an equal piece of the line.  A block's warps have equal parts of its tiles, one
// after the other.  Heads are not cut for a range kJoinTiles longer.
// Where the table has room for few tiles no head is cut, and the second kernel, which joins what several blocks had part in, not launched: it takes 4 us.
// kOneHead: one head of kWholeTiles at most (one head of 1000 rows of four 9.4 us, cut 10.0; 128 heads of up to 1500 11.9 and 12.8; 16 heads of up to 2000
// 15.6 and 11.0).  kTwoHeads: the i-th longest and the i-th last, of kMostSorted units, kPairTiles and twice as many heads as blocks at most (64 units of up to
// 1690 rows, 8 heads, 24.8, cut 29.4).  kHeadsInLine: more heads, of kLineTiles at most; a block has those that begin in its piece (320 units of up to 100 rows, 8
// heads, 18.2, cut 19.8).
constexpr int kWholeTiles = 24, kPairTiles = 32, kJoinTiles = 2 * kWarps, kSwitchTiles = kWarps, kMostSorted = 160, kLineTiles = 8;

__device__ __forceinline__ int unit_rows(const AttnArgs &A, int u) {
    const int n = A.rows[u], most = A.max_pages << A.page_shift;
    return n < 0 ? 0 : min(n, most);
}
__device__ __forceinline__ int tiles_of(int rows) { return (rows + kTile - 1) / kTile; }

struct Cut {
    int u0, u1, rows0, rows1;            // this lane's units, rows of the first two
    uint32_t mine, upto;                 // their tiles, of one head; with all units before
    uint32_t all, per, share;            // tiles of all heads; of a range, or 0; of a piece
    uint32_t ranges, ranges_upto;        // ranges of a head of each of this lane's units; with all units before
    __device__ __forceinline__ int rows(const AttnArgs &A, int u) const { return u == u0 ? rows0 : u == u0 + 1 ? rows1 : unit_rows(A, u); }
};
__device__ __forceinline__ uint32_t sum_upto(uint32_t x) {
    const int lane = lane_id();
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}
__device__ __forceinline__ Cut make_cut(const AttnArgs &A) {
    Cut c;
    const int each = (A.U + 31) >> 5;
    c.u0 = min(A.U, lane_id() * each);
    c.u1 = min(A.U, c.u0 + each);
    c.rows0 = c.u0 < c.u1 ? unit_rows(A, c.u0) : 0;
    c.rows1 = c.u0 + 1 < c.u1 ? unit_rows(A, c.u0 + 1) : 0;
    c.mine = tiles_of(c.rows0) + tiles_of(c.rows1);
    int longest = tiles_of(max(c.rows0, c.rows1));
#pragma unroll 1
    for (int u = c.u0 + 2; u < c.u1; ++u) {
        const int t = tiles_of(unit_rows(A, u));
        c.mine += t;
        longest = max(longest, t);
    }
    c.upto = sum_upto(c.mine);
    longest = __reduce_max_sync(0xFFFFFFFFu, longest);
    c.all = __shfl_sync(0xFFFFFFFFu, c.upto, 31) * A.Hkv;
    const uint32_t blocks = gridDim.x, heads = (uint32_t)A.U * A.Hkv;
    c.share = max(1u, (c.all + blocks - 1) / blocks);
    c.per = c.ranges = c.ranges_upto = 0;
    if (heads > blocks) return c;
    const uint32_t whole = max(1, longest);
#pragma unroll 1
    for (uint32_t per = c.share; per <= c.share + kSwitchTiles || per == whole; per += 2) {
        if (whole <= kWholeTiles || whole <= per + kJoinTiles) per = whole;
        uint32_t n = 0;
#pragma unroll 1
        for (int u = c.u0; u < c.u1; ++u) n += ((uint32_t)tiles_of(c.rows(A, u)) + per - 1) / per;
        if (__reduce_add_sync(0xFFFFFFFFu, n) * A.Hkv > blocks) continue;
        c.per = per;
        c.ranges = n;
        c.ranges_upto = sum_upto(n);
        break;
    }
    return c;
}
// A tile of the head (u, h): the unit's rows, and those from the tile's first one on.
struct Walk { int u, h, rows, left; };
struct Head { int u, h, rows; };
// On to the next tile; behind a block's first whole head comes its second one.
__device__ __forceinline__ void walk_on(const AttnArgs &A, Walk &w, const Head &second) {
    if ((w.left -= kTile) > 0) return;
    if (A.share == kTwoHeads) {
        w.u = second.u; w.h = second.h;
        w.rows = w.left = second.rows;
        return;
    }
    if (++w.h >= A.Hkv) {
        w.h = 0;
        do { ++w.u; w.rows = w.u < A.U ? unit_rows(A, w.u) : 0; } while (w.rows == 0 && w.u < A.U);
    }
    w.left = w.rows;
}
// A block's two whole heads, rows zero where there is none; kEach units a lane.  A unit's place is the number of units with more tiles, or with as many and a
// lower number, counted bit by bit over the warp: `same` are the units that are alike so far.
template <int kEach>
__device__ __forceinline__ void two_heads(const AttnArgs &A, Head &first, Head &second) {
    const int lane = lane_id();
    int rows[kEach], place[kEach];
    uint32_t same[kEach][kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        rows[i] = lane + 32 * i < A.U ? unit_rows(A, lane + 32 * i) : 0;
        place[i] = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) same[i][k] = ~0u;
    }
    static_assert(kPairTiles < 64, "six bits");
#pragma unroll 1
    for (int b = 5; b >= 0; --b) {
        uint32_t has[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) has[k] = __ballot_sync(0xFFFFFFFFu, tiles_of(rows[k]) >> b & 1);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t turn = tiles_of(rows[i]) >> b & 1 ? 0u : ~0u;      // units with the bit are before one without it; then alike are those with the same
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                place[i] += __popc(same[i][k] & has[k] & turn);
                same[i][k] &= has[k] ^ turn;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
#pragma unroll
        for (int k = 0; k < i; ++k) place[i] += __popc(same[i][k]);
        place[i] += __popc(same[i][i] & lanemask_lt());
    }
    auto find = [&](uint32_t number, Head &head) {
        head = {0, 0, 0};
        if (number >= (uint32_t)A.U * A.Hkv) return;
        const int at = A.by_heads.div(number);
        head.h = number - at * A.Hkv;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t here = __ballot_sync(0xFFFFFFFFu, place[i] == at);
            const int owner = __ffs(here) - 1, n = __shfl_sync(0xFFFFFFFFu, rows[i], owner & 31);
            if (here) { head.u = owner + 32 * i; head.rows = n; }
        }
    };
    find(blockIdx.x, first);
    find(2 * gridDim.x - 1 - blockIdx.x, second);
}
// Where tile x is, x below c.all.
__device__ __forceinline__ Walk walk_to(const AttnArgs &A, const Cut &c, uint32_t x) {
    const uint32_t H = A.Hkv;
    const int owner = __ffs(__ballot_sync(0xFFFFFFFFu, x < c.upto * H)) - 1;
    int u = 0, rows = 0;
    uint32_t base = 0;                                                // tiles of a head of each of the units before
    if (lane_id() == owner) {
        base = c.upto - c.mine;
#pragma unroll 1
        for (u = c.u0;; ++u) {
            rows = c.rows(A, u);
            const int t = tiles_of(rows);
            if (u == c.u1 - 1 || x < (base + t) * H) break;
            base += t;
        }
    }
    Walk w;
    w.u = __shfl_sync(0xFFFFFFFFu, u, owner);
    w.rows = __shfl_sync(0xFFFFFFFFu, rows, owner);
    base = __shfl_sync(0xFFFFFFFFu, base, owner) * H;
    const uint32_t tiles = tiles_of(w.rows);
    w.h = (x - base) / tiles;
    w.left = w.rows - (int)(x - base - w.h * tiles) * kTile;
    return w;
}
// The block's tiles [x0, x1); none: x0 == x1.
__device__ __forceinline__ void block_piece(const AttnArgs &A, const Cut &c, uint32_t &x0, uint32_t &x1) {
    if (c.per == 0) {
        x0 = min(c.all, blockIdx.x * c.share);
        x1 = min(c.all, x0 + c.share);
        if (A.share == kHeadsInLine) {
            auto head = [&](uint32_t x) {                            // the first head's tile from x on
                if (x >= c.all) return x;
                const Walk w = walk_to(A, c, x);
                const int done = (w.rows - w.left) / kTile;
                return done ? x + tiles_of(w.rows) - done : x;
            };
            x0 = head(x0);
            x1 = head(x1);
        }
        return;
    }
    // ranges are numbered by unit, head and key
    const uint32_t H = A.Hkv, i = blockIdx.x, hit = __ballot_sync(0xFFFFFFFFu, i < c.ranges_upto * H);
    x0 = x1 = 0;
    if (hit == 0) return;
    const int owner = __ffs(hit) - 1;
    if (lane_id() == owner) {
        uint32_t ranges = (c.ranges_upto - c.ranges) * H, base = (c.upto - c.mine) * H;
#pragma unroll 1
        for (int u = c.u0; u < c.u1; ++u) {
            const uint32_t t = tiles_of(c.rows(A, u)), n = (t + c.per - 1) / c.per;
            if (i < ranges + n * H) {
                const uint32_t in = i - ranges, h = in / n, first = (in - h * n) * c.per;
                x0 = base + h * t + first;
                x1 = x0 + min(c.per, t - first);
                break;
            }
            ranges += n * H;
            base += t * H;
        }
    }
    x0 = __shfl_sync(0xFFFFFFFFu, x0, owner);
    x1 = __shfl_sync(0xFFFFFFFFu, x1, owner);
}

// ---- matrix instructions -------------------------------------------------------------------------
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {      // onto zeros
    asm("{\n\t.reg .f32 z;\n\tmov.f32 z, 0f00000000;\n\t"
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {z, z, z, z};\n\t}"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 by 8 matrix of fp16, a row of it in four neighbouring lanes, transposed; by a whole warp.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    uint32_t h;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
    return h;
}
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) {
    uint32_t h;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(h) : "r"(a), "r"(b));
    return h;
}
// both halves times one half of b (which the instruction picks by itself)
__device__ __forceinline__ uint32_t times_one(uint32_t a, uint32_t b, int upper) {
    const __half2 x = *reinterpret_cast<const __half2 *>(&a), y = *reinterpret_cast<const __half2 *>(&b), z = __hmul2_rn(x, upper ? __high2half2(y) : __low2half2(y));
    return *reinterpret_cast<const uint32_t *>(&z);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max_over_rows(float x) {              // over the lanes with the same lane % 4
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

// The query operand of a head: a lane has query head lane / 4, the channels that it takes of a K row, and of every word of eight the pairs in order.
template <int D, bool kTwo> struct Queries {
    uint32_t hi[D / 8], lo[kTwo ? D / 8 : 1];      // [D / 32 words][4 pairs]
    float factor[2];                               // of the logits of query heads 2 (lane % 4) and the next one
};
template <typename T, int D>
__device__ __forceinline__ void load_queries(const AttnArgs &A, int u, int h, Queries<D, sizeof(T) == 4> &Q) {
    constexpr bool kTwo = sizeof(T) == 4;
    constexpr int kWords = D / 32;
    const int lane = lane_id(), r = lane >> 2, t = lane & 3;
    const T *q = static_cast<const T *>(A.q) + ((int64_t)u * A.Hq + h * A.G + r) * D + t * (D / 4);
    Eight<T> raw[kWords];
    uint32_t size = 0;
    const bool on = r < A.G;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        if (on) {
            raw[w].load(q + 8 * w);
            size = max(size, raw[w].size());
        }
    }
    size = max(size, __shfl_xor_sync(0xFFFFFFFFu, size, 1));
    size = max(size, __shfl_xor_sync(0xFFFFFFFFu, size, 2));
    const bool finite = size < paged::kInfinityBits;
    const int ex = finite ? max(-100, (int)(size >> 23) - 127) - 14 : 0;          // the largest element to [2^14, 2^15)
    const float f = paged::power_of_two(-ex);
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        float x[8];
        if (on) raw[w].get(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = on ? x[2 * i] * f : 0.f, b = on ? x[2 * i + 1] * f : 0.f;
            const uint32_t hi = half2_of(a, b);
            Q.hi[4 * w + i] = hi;
            if constexpr (kTwo) {
                const float2 g = from_half2(hi);
                Q.lo[4 * w + i] = half2_of(a - g.x, b - g.y);
            }
        }
    }
    const float factor = finite ? fmaxf(paged::power_of_two(ex) * A.scale_log2, 1.175494351e-38f) : __uint_as_float(0x7FC00000u);     // (not zero: times -inf)
    Q.factor[0] = __shfl_sync(0xFFFFFFFFu, factor, 8 * t);
    Q.factor[1] = __shfl_sync(0xFFFFFFFFu, factor, 8 * t + 4);
}

// ---- records -------------------------------------------------------------------------------------
// [heads][D] outputs relative to the maximum, then maxima (log2), then sums of weights; 16 neighbouring channels of two query heads a lane (D = 64: eight).
template <int D>
__device__ __forceinline__ void put_record(float *rec, const float (&o)[D / 16][4], const float (&m)[2], const float (&l)[2]) {
    const int lane = lane_id(), r = lane >> 2, t = lane & 3;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float4 *to = reinterpret_cast<float4 *>(rec + (2 * t + q) * D + r * (D / 8));
#pragma unroll
        for (int j = 0; j < D / 16; j += 2) to[j / 2] = make_float4(o[j][q], o[j][2 + q], o[j + 1][q], o[j + 1][2 + q]);
        if (r == 0) { rec[kHeads * D + 2 * t + q] = m[q]; rec[kHeads * (D + 1) + 2 * t + q] = l[q]; }
    }
}
__device__ __forceinline__ void put_four(float *to, const float (&x)[4]) { *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void put_four(__nv_bfloat16 *to, const float (&x)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void put_eight(float *to, const float (&x)[8]) {
    reinterpret_cast<float4 *>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void put_eight(__nv_bfloat16 *to, const float (&x)[8]) { Elem<__nv_bfloat16>::store16(to, x); }

// What the parts of heads at both ends of a warp's tiles are: the first part's head began before them (a front), and ends in them; the last part's head
// begins in them and goes on (a back).
constexpr int kFront = 1, kEnds = 2, kBack = 4;
struct Meta {
    int flags;
    int fu, fh, bu, bh;                  // the heads of front and back
    int blocks;                          // that have part in the back's head, should it go on behind this block
};
static_assert(sizeof(Meta) <= 32, "as much as Lay::kMeta leaves");

// kLong: pages of kTile rows and more, so that a tile is on one page.
template <typename T, int D, bool kLong>
__global__ void __launch_bounds__(kAttnThreads, kBlocks) nibble_attention_kernel(const AttnArgs A) {
    typedef Lay<D> L;
    constexpr bool kTwo = sizeof(T) == 4;
    constexpr float kWeightExponent = kTwo ? 14.f : 10.f;
    constexpr int kWords = D / 32, kSubs = kTile / 16;               // words of a K row that a lane has; subtiles of 16 keys
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
    uint8_t *ring = smem + warp * (3 * L::kHalf);
    float *record = reinterpret_cast<float *>(smem + L::kRecords + warp * L::kRecord);
    Meta *meta = reinterpret_cast<Meta *>(smem + L::kMeta);
    predecessor_done();
    successor_may_start();
    // lengths out of range, units without rows (while the first tiles are on their way)
    auto aside = [&]() {
        if (blockIdx.x == 0)
#pragma unroll 1
            for (int u = threadIdx.x; u < A.U; u += kAttnThreads) {
                const int n = A.rows[u];
                if (n < 0 || n > A.max_pages << A.page_shift) report(A.status, kStatusIndex);
            }
#pragma unroll 1
        for (int u = blockIdx.x * kWarps + warp; u < A.U; u += gridDim.x * kWarps)
            if (unit_rows(A, u) == 0)
#pragma unroll 1
                for (int i = lane; i < A.Hq * D / 4; i += 32) {
                    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
                    put_four(static_cast<T *>(A.out) + (int64_t)u * A.Hq * D + 4 * i, zero);
                }
    };
    // One head: the table is read together with the length.  Two, or a piece of the line: the lengths say what the block has.
    Cut cut;
    Walk cur;
    Head whole, second = {0, 0, 0};
    uint32_t x0 = 0, x1;
    int ids = 0, ids_unit = -1, ids_base = 0;                        // 32 entries of the block table
    if (A.share <= kTwoHeads) {
        if (A.share == kTwoHeads) {
            if (A.U <= 64) two_heads<2>(A, whole, second);
            else two_heads<kMostSorted / 32>(A, whole, second);
        } else {
            whole.u = ids_unit = A.by_heads.div(blockIdx.x);
            whole.h = blockIdx.x - whole.u * A.Hkv;
            whole.rows = unit_rows(A, whole.u);
            ids = lane < A.max_pages ? A.table[(int64_t)whole.u * A.max_pages + lane] : 0;
            if (lane >= (whole.rows + (1 << A.page_shift) - 1) >> A.page_shift) ids = 0;
            if ((unsigned)ids >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); ids = 0; }
        }
        x1 = tiles_of(whole.rows) + tiles_of(second.rows);
    } else {
        cut = make_cut(A);
        block_piece(A, cut, x0, x1);
    }
    const uint32_t each = (x1 - x0 + kWarps - 1) / kWarps;
    const uint32_t w0 = min(x1, x0 + warp * each), w1 = min(x1, w0 + each);
    const int count = (int)(w1 - w0);
    Meta me = {0, 0, 0, 0, 0, 0};
    if (count > 0) {
        // Copies of 16 bytes, a lane the codes of row lane / kLanes of every kRows of the tile, and scales that lie side by side.  Sixteen rows are on one
        // page and come or are left out together.
        constexpr int kLanes = D / 32, kRows = 32 / kLanes, kScaleRows = 256 / D;
        const int page = 1 << A.page_shift, scale_group = lane * kScaleRows >> 4;
        const uint32_t to = tc::smem_u32(ring) + lane * 16, page_rows = (uint32_t)A.Hkv << A.page_shift;
        // where the tile's codes are, from this lane's first sixteen bytes on, for every sixteen rows; the lane's scales; the tile's rows
        struct Source { int64_t codes[kLong ? 1 : kTile / 16], scales; int left; } next;
        auto locate = [&](const Walk &w) {
            const int at = w.rows - w.left, first = at >> A.page_shift;
            if (w.u != ids_unit || (first & ~31) != ids_base) {
                ids_unit = w.u;
                ids_base = first & ~31;
                const int p = ids_base + lane;
                ids = p < (w.rows + page - 1) >> A.page_shift ? A.table[(int64_t)w.u * A.max_pages + p] : 0;
                if ((unsigned)ids >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); ids = 0; }
            }
            next.left = w.left;
            auto row = [&](int of) {                                 // the number in the pool of the tile's row `of`
                return (int64_t)((uint64_t)(uint32_t)__shfl_sync(0xFFFFFFFFu, ids, first + (of >> A.page_shift)) * page_rows) +
                       (uint32_t)((w.h << A.page_shift) + ((at + of) & (page - 1)));
            };
            if constexpr (kLong) {
                const int64_t r0 = row(0);
                next.codes[0] = r0 * (D / 2) + lane * 16;
                next.scales = r0 * (D / kGroup) + lane * 16;
            } else {
#pragma unroll
                for (int g = 0; g < kTile / 16; ++g) next.codes[g] = row(16 * g) * (D / 2) + lane * 16;
                next.scales = row(lane * kScaleRows) * (D / kGroup);
            }
        };
        uint32_t put = 0;                                            // the ring's next place
        auto issue = [&](int which, bool on) {
            if (on) {
                const uint32_t there = to + put * L::kHalf;
                auto copy = [&](int g) {
                    const uint8_t *codes = A.pages[which] + (kLong ? next.codes[0] + g * (8 * D) : next.codes[kLong ? 0 : g]);
#pragma unroll
                    for (int i = 0; i < 16 / kRows; ++i) tc::copy16_async(there + g * (8 * D) + i * 512, codes + i * 512);
                };
                if (next.left >= kTile) {
#pragma unroll
                    for (int g = 0; g < kTile / 16; ++g) copy(g);
                    if (kTile == 32 * kScaleRows || lane < kTile / kScaleRows) tc::copy16_async(there + L::kCodes, A.scale[which] + next.scales);
                } else {
#pragma unroll
                    for (int g = 0; g < kTile / 16; ++g)
                        if (16 * g < next.left) copy(g);
                    if (lane < kTile / kScaleRows && 16 * scale_group < next.left) tc::copy16_async(there + L::kCodes, A.scale[which] + next.scales);
                }
            }
            tc::copies_commit();
            put = put == 2 ? 0 : put + 1;
        };
        if (A.share <= kTwoHeads) {
            const int at = (int)w0 - tiles_of(whole.rows);            // in the second head
            const Head &of = at < 0 ? whole : second;
            cur = {of.u, of.h, of.rows, of.rows - (at < 0 ? (int)w0 : at) * kTile};
        } else {
            cur = walk_to(A, cut, w0);
        }
        Walk far = cur;
        uint32_t take = 0;
        locate(far);
        issue(0, true);
        issue(1, true);
        if (count > 1) { walk_on(A, far, second); locate(far); }
        issue(0, count > 1);
        aside();
        Queries<D, kTwo> Q;
        float o[D / 16][4];
        float2 l, minus;                                             // sums of weights, of this lane's keys; the references, their signs turned
        bool fresh = true;                                           // a part of a head begins
        bool begins = true;                                          // ... with the head's first row
        for (int i = 0; i < count; ++i) {
            if (fresh) {
                load_queries<T, D>(A, cur.u, cur.h, Q);
                begins = cur.left == cur.rows;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
                minus.x = minus.y = __uint_as_float(0x7F800000u);    // (the first product is above it)
                l = make_float2(0.f, 0.f);
                fresh = false;
            }
            const int valid = cur.left;                              // rows, should they be fewer than a tile's
            tc::copies_wait<2>();                                    // (of three half tiles on their way)
            __syncwarp();
            // products with keys: a lane's rows of a subtile are keys `key` and key + 8, its columns query heads 2 t and 2 t + 1
            const int key = r ^ (r >> 1 & 1);
            float z[kSubs][4];
            {
                const uint8_t *codes = ring + take * L::kHalf + key * (D / 2) + t * (D / 8), *scales = ring + take * L::kHalf + L::kCodes + key * (D / 16) + t * (D / 64);
#pragma unroll
                for (int s = 0; s < kSubs; ++s) {
                    uint32_t w[2][kWords], sc[2];                    // [8 further], scales of the first two words and the next
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int row = 16 * s + 8 * b;
                        if constexpr (D == 128) {
                            const uint4 v = *reinterpret_cast<const uint4 *>(codes + row * 64);
                            w[b][0] = v.x; w[b][1] = v.y; w[b][kWords - 2] = v.z; w[b][kWords - 1] = v.w;
                            const uint32_t both = *reinterpret_cast<const unsigned short *>(scales + row * 8);
                            sc[b] = __byte_perm(both, 0, 0x4140) << 7;
                        } else {
                            const uint2 v = *reinterpret_cast<const uint2 *>(codes + row * 32);
                            w[b][0] = v.x; w[b][1] = v.y;
                            sc[b] = (uint32_t)scales[row * 4] << 7;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kWords; ++j) {
                        uint32_t lo[4], hi[4];
                        widen8(w[0][j], lo);
                        widen8(w[1][j], hi);
#pragma unroll
                        for (int p = 0; p < 4; ++p) { lo[p] = times_one(lo[p], sc[0], j >> 1); hi[p] = times_one(hi[p], sc[1], j >> 1); }
#pragma unroll
                        for (int p = 0; p < 4; p += 2) {
                            const uint32_t a[4] = {lo[p], hi[p], lo[p + 1], hi[p + 1]};
                            if (j == 0 && p == 0) mma_first(z[s], a, Q.hi[0], Q.hi[1]);
                            else mma(z[s], a, Q.hi[4 * j + p], Q.hi[4 * j + p + 1]);
                            if constexpr (kTwo) mma(z[s], a, Q.lo[4 * j + p], Q.lo[4 * j + p + 1]);
                        }
                    }
                }
            }
            __syncwarp();
            issue(1, i + 1 < count);                                 // the next tile's V, where this one's K was
            take = take == 2 ? 0 : take + 1;
            if (valid < kTile) {
#pragma unroll
                for (int s = 0; s < kSubs; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (16 * s + 8 * (e >> 1) + key >= valid) z[s][e] = __uint_as_float(0xFF800000u);
            }
            float top[2] = {fmaxf(z[0][0], z[0][2]), fmaxf(z[0][1], z[0][3])};
#pragma unroll
            for (int s = 1; s < kSubs; ++s) {
                top[0] = max3(top[0], z[s][0], z[s][2]);
                top[1] = max3(top[1], z[s][1], z[s][3]);
            }
            constexpr float kRoom = kMostExponent - kWeightExponent;
            if (__any_sync(0xFFFFFFFFu, (top[0] + minus.x) * Q.factor[0] > kRoom || (top[1] + minus.y) * Q.factor[1] > kRoom)) {
                const float2 next = make_float2(fminf(-max_over_rows(top[0]), minus.x), fminf(-max_over_rows(top[1]), minus.y));
                const float c[2] = {tc::ex2((next.x - minus.x) * Q.factor[0]), tc::ex2((next.y - minus.y) * Q.factor[1])};
                minus = next;
                l = tc::fmul2(l, make_float2(c[0], c[1]));
#pragma unroll
                for (int j = 0; j < D / 16; ++j) { o[j][0] *= c[0]; o[j][1] *= c[1]; o[j][2] *= c[0]; o[j][3] *= c[1]; }
            }
            tc::copies_wait<2>();                                    // (of three half tiles on their way)
            __syncwarp();
            if (valid < kTile) {                                     // what stands behind the last row counts for nothing, NaN neither
                uint8_t *scales = ring + take * L::kHalf + L::kCodes;
#pragma unroll 1
                for (int b = valid * (D / 16) + lane; b < (int)L::kScales; b += 32) scales[b] = 0;
                __syncwarp();
            }
            {
                const int ka = 2 * t ^ (t & 1), kb = (2 * t + 1) ^ (t & 1);      // the keys at places 2 t and 2 t + 1
                const uint8_t *codes = ring + take * L::kHalf + r * (D / 16), *scales = ring + take * L::kHalf + L::kCodes + (D == 128 ? r : r >> 1);
                const uint8_t *codes_of[2] = {codes + ka * (D / 2), codes + kb * (D / 2)}, *scales_of[2] = {scales + ka * (D / 16), scales + kb * (D / 16)};
                const float2 factor = make_float2(Q.factor[0], Q.factor[1]), most = make_float2(kWeightExponent, kWeightExponent);
#pragma unroll
                for (int s = 0; s < kSubs; ++s) {
                    uint32_t p[2], q[2];                             // weights of keys at places 0 to 7 and 8 to 15; their rests
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float2 x = tc::ffma2(tc::fadd2(make_float2(z[s][2 * b], z[s][2 * b + 1]), minus), factor, most);
                        x = make_float2(tc::ex2(x.x), tc::ex2(x.y));
                        l = tc::fadd2(l, x);
                        p[b] = half2_of(x.x, x.y);
                        if constexpr (kTwo) {
                            const float2 h = from_half2(p[b]);
                            q[b] = transposed(half2_of(x.x - h.x, x.y - h.y));
                        }
                        p[b] = transposed(p[b]);
                    }
                    // V's operand: even and odd channels, [places 2 t, 2 t + 1 | 8 further], a pair of keys in a register
                    uint32_t w[2][2][D / 64], sc[2];                  // [8 further][key][words]
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int row = 16 * s + 8 * b;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if constexpr (D == 128) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(codes_of[k] + row * 64);
                                w[b][k][0] = v.x; w[b][k][D / 64 - 1] = v.y;
                            } else {
                                w[b][k][0] = *reinterpret_cast<const uint32_t *>(codes_of[k] + row * 32);
                            }
                        }
                        sc[b] = scales_of[0][row * (D / 16)] * 0x00000080u + scales_of[1][row * (D / 16)] * 0x00800000u;
                    }
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        uint32_t even[2][4], odd[2][4];
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const uint32_t x = w[b][0][j], y = w[b][1][j];
                            widen8((x & 0x0F0F0F0Fu) | (y << 4 & 0xF0F0F0F0u), even[b]);
                            widen8((x >> 4 & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u), odd[b]);
#pragma unroll
                            for (int k = 0; k < 4; ++k) { even[b][k] = times(even[b][k], sc[b]); odd[b][k] = times(odd[b][k], sc[b]); }
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t a[4] = {even[0][k], odd[0][k], even[1][k], odd[1][k]};
                            float(&sum)[4] = o[4 * j + k];
                            if constexpr (kTwo) {
                                // (a matrix instruction cuts off what it adds to, always towards zero: a line of them onto the same sums was off by 3e-6 after 64
                                // tiles, by 2.4e-5 after 112 of values above zero, so a subtile's products are summed by themselves and added to the nearest; 4
                                // to 8 % of the time.  A tile's summed so, weights first: 13 % for 128 channels, 3 % for 64.)
                                float own[4];
                                mma_first(own, a, q[0], q[1]);
                                mma(own, a, p[0], p[1]);
                                const float2 x = tc::fadd2(make_float2(sum[0], sum[1]), make_float2(own[0], own[1])), y = tc::fadd2(make_float2(sum[2], sum[3]), make_float2(own[2], own[3]));
                                sum[0] = x.x; sum[1] = x.y; sum[2] = y.x; sum[3] = y.y;
                            } else {
                                mma(sum, a, p[0], p[1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            take = take == 2 ? 0 : take + 1;
            if (i + 2 < count) { walk_on(A, far, second); locate(far); }
            issue(0, i + 2 < count);                                 // K of the tile after the next one, where this one's V was
            const bool last = cur.left <= kTile;
            if (last || i + 1 == count) {                            // the part ends
                float sum[2] = {l.x, l.y};
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) sum[q] += __shfl_xor_sync(0xFFFFFFFFu, sum[q], k);
                // (a record's maximum: all weights of a head are 2^10 for a logit at it, or all 2^14; equal products have equal ones)
                const float most[2] = {-minus.x * Q.factor[0], -minus.y * Q.factor[1]};
                if (begins && last) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if (2 * t + q >= A.G) continue;
                        const float inverse = reciprocal(sum[q]);
                        T *out = static_cast<T *>(A.out) + ((int64_t)cur.u * A.Hq + cur.h * A.G + 2 * t + q) * D + r * (D / 8);
#pragma unroll
                        for (int j = 0; j < D / 16; j += 2) {
                            const float x[4] = {o[j][q] * inverse, o[j][2 + q] * inverse, o[j + 1][q] * inverse, o[j + 1][2 + q] * inverse};
                            put_four(out + 2 * j, x);
                        }
                    }
                } else if (!begins) {
                    me.flags |= last ? kFront | kEnds : kFront; me.fu = cur.u; me.fh = cur.h;
                    put_record<D>(record, o, most, sum);
                } else {
                    me.flags |= kBack; me.bu = cur.u; me.bh = cur.h;
                    const uint32_t tiles = tiles_of(cur.rows), done = (cur.rows - cur.left) / kTile;
                    if (A.share == kCutHeads) me.blocks = cut.per ? (tiles + cut.per - 1) / cut.per : (w0 + i - done + tiles - 1) / cut.share - blockIdx.x + 1;
                    put_record<D>(reinterpret_cast<float *>(ring), o, most, sum);       // (no copy is on its way any more)
                }
                fresh = true;
            }
            walk_on(A, cur, second);
        }
    }
    if (count == 0) aside();
    if (lane == 0) meta[warp] = me;
    __syncthreads();
    int4 note = make_int4(0, 0, 0, 0);
    if (x1 > x0) {
        // Heads that several warps had part in: a chain of records, from a back, or from the block's first front, on to the front that ends.  A thread has
        // eight channels of a query head, and all their records on their way at once.
        const int flags = lane < kWarps ? meta[lane].flags : 0;
        const uint32_t fronts = __ballot_sync(0xFFFFFFFFu, flags & kFront), ending = __ballot_sync(0xFFFFFFFFu, flags & kEnds),
                       backs = __ballot_sync(0xFFFFFFFFu, flags & kBack);
#pragma unroll 1
        for (uint32_t starts = (fronts & 1u) | backs << 1; starts; starts &= starts - 1u) {
            const int from = __ffs(starts) - 1, back = from - 1;     // the chain's first front; the warp that has its back, -1: none, it began in a block before
            const int end = from + __ffs((~fronts | (ending << 1 & ~1u << from)) >> from) - 1;      // fronts: of warps from, ..., end - 1
            const bool ends = end > from && (ending >> (end - 1) & 1u);
            const int u = back < 0 ? meta[0].fu : meta[back].bu, h = back < 0 ? meta[0].fh : meta[back].bh;
            if (back >= 0 && !ends) note = make_int4(u, h * A.G, meta[back].blocks, A.G);            // (it goes on in the next block)
            const int g = threadIdx.x / (D / 8), d = threadIdx.x % (D / 8) * 8;
            static_assert(kHeads * (D / 8) <= kAttnThreads, "eight channels a thread");
            if (g >= A.G) continue;
            float tops[kWarps], sums[kWarps], top = kLowest, sum = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            float4 part[kWarps][2];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float *rec = reinterpret_cast<const float *>(w == back ? smem + w * (3 * L::kHalf) : smem + L::kRecords + w * L::kRecord);
                const bool on = w == back || (w >= from && w < end);
                tops[w] = on ? rec[kHeads * D + g] : kLowest;
                sums[w] = on ? rec[kHeads * (D + 1) + g] : 0.f;
#pragma unroll
                for (int k = 0; k < 2; ++k) part[w][k] = on ? *reinterpret_cast<const float4 *>(rec + g * D + d + 4 * k) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, tops[w]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float c = tc::ex2(tops[w] - top);
                sum = fmaf(sums[w], c, sum);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[4 * k] = fmaf(part[w][k].x, c, x[4 * k]); x[4 * k + 1] = fmaf(part[w][k].y, c, x[4 * k + 1]);
                    x[4 * k + 2] = fmaf(part[w][k].z, c, x[4 * k + 2]); x[4 * k + 3] = fmaf(part[w][k].w, c, x[4 * k + 3]);
                }
            }
            if (back >= 0 && ends) {
                const float inverse = reciprocal(sum);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] *= inverse;
                put_eight(static_cast<T *>(A.out) + ((int64_t)u * A.Hq + h * A.G + g) * D + d, x);
            } else {
                float *out = A.part + (int64_t)(2 * blockIdx.x + (back >= 0)) * paged::record_floats(A.G, D);
                put_eight(out + g * D + d, x);
                if (d == 0) { out[A.G * D + g] = top; out[A.G * (D + 1) + g] = sum; }
            }
        }
    }
    if (A.cut_heads && threadIdx.x == 0) A.cut_heads[blockIdx.x] = note;
}

}  // namespace nibble
}  // namespace flowmm
