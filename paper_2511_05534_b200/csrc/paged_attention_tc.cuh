// Decode attention over the paged 8-bit cache on the tensor cores: bf16 queries.
//
// The codes go into the matrix instructions as they are (kind::f8f6f4), with the keys on the wide side, so no code is ever
// converted and every row of K and V is read once.  The narrow side is split into e4m3 numbers that stand side by side as columns:
//   S[key, head]: a bf16 query, scaled by a power of two, is the sum of two e4m3 numbers, 8 bits of significand as 4 + 4 (exact but
//                 for elements 2^13 times smaller than the largest): N = 8 heads x 2
//   O[dim, head]: a weight is kept as four e4m3 numbers, each the rounded rest of the one before times 16, within 2^-16 of
//                 itself or 2^-30 of the largest: N = 8 heads x 4.  (Two would do for a bf16 result; the time without any splitting is 1 % less where memory bounds.)
// The pages' scales join in fp32: K's on the logits; V's in the exponent of the weights, w_j = 2^(z_j + log2 sv_j - max), with a maximum of
// its own, so that the largest weight is 1 whatever the scales are.  The sum of the softmax, sum_j 2^(z_j - max z), is apart.  The second maximum is held as
// what it is above the first, and weights are formed from z_j - max z, a number of its own size: log2 sv_j would be lost next to logits of 2^24.
//
// How the work is shared out over the blocks of the launch, two to an SM, is found on the device, where alone the lengths are known (Cut).
// Few heads: a block has one range of one head, all of the same length but for a head's last one.  Many: a block has two whole heads, or the
// tiles of 128 keys of all heads stand in a row, by unit, head and key, and every block takes an equal piece of the row, parts of heads or
// several, one after the other.  A head that several blocks have part in leaves a record for each, and cache_join_kernel joins
// them in order.  (Ranges alone left a last round half empty, 16 sequences of up to 33 792 rows, 8 heads, 174 us when pieces took 118.  Three
// quarters of a piece to each block and the rest drawn from a counter in pieces of three tiles and more: 132 then.)
// A block goes through its tiles in groups of up to seven of one head, the roles of its warps one or two groups apart, across the
// heads' borders too:
//   warp 0     K tiles and V tiles by TMA, a box per page, into a ring of six stages of 16 KB (ten of 8): a tile of K of group c + 1 and one of V of
//              group c in turn; the scales of a group's pages
//   warp 1     the products, in the same order; the logits of two groups stay in tensor memory
//   warps 2-9  a thread per key of a tile: maxima of a group, then its weights; a thread per dim: the output, rescaled once a group; a warp per query
//              head: the next head's query operand.
//              Two halves of four warps: for more than four query heads each has four of them, for fewer every other tile.  (One half
//              alone took 1800 clocks for a tile of eight heads, longer than its share of the memory's time.)
// Memory bounds long calls: 16 sequences of up to 33 792 rows, 654 MB of pages, 107 us, 6.1 TB/s.  Short ones are bound by the way of one group through the
// block, about 6 us from the lengths to the output (one sequence of 218 rows), and by the ends of the blocks, which fall together: 64
// sequences of up to 1690 rows, 129 MB, 34.5 us.  (Groups of two to five tiles, and smaller groups at a block's end, were no faster.)
// Every wait is bounded.
#pragma once
#include "paged_attention.cuh"

namespace flowmm {
namespace paged {
namespace ptc {

constexpr int kTile = 128, kMaxHeads = 8, kHalf = 4, kGroup = 7, kThreads = 320, kTmemCols = 256;
constexpr int kQCols = 2 * kMaxHeads, kPCols = 4 * kMaxHeads;            // N of the two products; by half, piece, head
constexpr int kMostPages = kGroup * kTile / 16;                          // pages of a group
constexpr int kInfos = 4;                                                // groups whose scales are kept
constexpr int kInfo = 2 * kMostPages;                                     // [K's scale, log2 of V's][page]
constexpr float kFar = 1048576.f;                                         // a logit (log2) beyond which V's scales are not added to it
constexpr uint32_t kPBytes = kTile * kPCols;                              // the weights of a tile
constexpr uint32_t kColS = kPCols;                                        // O in the first columns, then the two groups' logits
static_assert(kColS + 2 * kGroup * kQCols <= kTmemCols, "tensor memory");

// What goes by the heads' dims: the ring (of 96 or 80 KB), the rows of tiles and query operands, in the swizzle of their length, and the
// places of it all in shared memory.
template <int D> struct Lay {
    static constexpr int kStages = D == 128 ? 6 : 10;
    static constexpr uint32_t kStageBytes = kTile * D, kQBytes = kQCols * D;
    static constexpr uint32_t kSmemQ = kStages * kStageBytes, kSmemP = kSmemQ + 2 * kQBytes, kSmemRed = kSmemP + 2 * kPBytes;
    static constexpr uint32_t kSmemInfo = kSmemRed + 2 * 8 * 3 * kHalf * 4;   // red: [group parity][warp][maxima, with V's scales, sums][head]
    static constexpr uint32_t kSmemFactor = kSmemInfo + kInfos * kInfo * 4;   // the factors of the queries: [head mod 2]
    static constexpr uint32_t kSmemTask = kSmemFactor + 2 * kMaxHeads * 4;    // tasks: [group mod 4]
    static constexpr uint32_t kSmemBar = kSmemTask + kInfos * 32;
    static constexpr int kBarFull = 0, kBarEmpty = kStages, kBarQFull = 2 * kStages,
        kBarS = kBarQFull + 2 /* a tile's logits, by its number in the block */, kBarPFull = kBarS + 2 * kGroup, kBarPEmpty = kBarPFull + 2,
        kBarO = kBarPEmpty + 2, kBarTask = kBarO + 1, kBarIFull = kBarTask + kInfos, kBarIEmpty = kBarIFull + kInfos, kNumBars = kBarIEmpty + kInfos;
    static constexpr uint32_t kSmemBytes = kSmemBar + 8 * kNumBars + 16;      // (+ TMEM address, abort flag, status)
    static_assert(2 * (kSmemBytes + 1024) <= 227 * 1024, "two blocks to an SM");
    // rows of 128 bytes in the 128-byte swizzle, of 64 in the 64-byte one, groups of eight rows one after the other
    static constexpr uint32_t kDescHi = D == 128 ? tc::kDescSw128Hi : (512u >> 4) | (1u << 14) | (4u << 29);
    // where 16 bytes of a row go
    static __device__ __forceinline__ uint32_t chunk(int row, int c) { return (uint32_t)(row * D + ((D == 128 ? c ^ (row & 7) : c ^ (row >> 1 & 3)) << 4)); }
};

__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N) { return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24); }
constexpr uint32_t kIdescQK = idesc_e4m3(kTile, kQCols);
// The second product's operands have the contraction's index, the key, as rows: V a row of dims (M) as it came, the weights a row of 32
// (N) in the 32-byte swizzle, groups of eight rows 256 bytes apart; so a thread writes its key's weights of four heads with one store.
// M is 128 for heads of 64 as well: the next 64 dims are said to be 0 bytes further on, are the first ones again, and are not looked at.
constexpr uint32_t kIdescPV = idesc_e4m3(128, kPCols) | 1u << 15 | 1u << 16;
constexpr uint32_t kDescPHi = (256u >> 4) | (1u << 14) | (6u << 29);

// D[tmem] (+)= A[smem] B[smem]^T, e4m3 inputs, fp32 accumulate; one thread issues.
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 a, {%1, %2};\n\t"
        "mov.b64 b, {%3, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 8 consecutive fp32 columns of this thread's TMEM lane, and the wait tied to them (so that a load may stay on its way across other work).
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(float (&r)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7])
                 :
                 : "memory");
}
// The largest of a warp's values (NaN counts for nothing).
__device__ __forceinline__ float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));      // (volatile: not to be moved to where one lane alone needs it)
    return y;
}
// The epilogue's warps meet; whether all of them go on.  (A wait may run out for one warp and not for another: then all leave here.)
__device__ __forceinline__ bool epi_all(bool ok) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.and.pred q, 1, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all)
        : "r"((uint32_t)ok)
        : "memory");
    return all != 0;
}
__device__ __forceinline__ void sts128(uint32_t addr, const uint32_t (&v)[4]) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t v) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"((unsigned short)v) : "memory"); }
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float log2_of(float x) {
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x in [0, 256] as four e4m3 numbers, p0 + p1 / 16 + p2 / 256 + p3 / 4096, for two x at once; each piece two codes
__device__ __forceinline__ void four_pieces(float2 x, uint32_t (&piece)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        piece[i] = to_e4m3x2(x.x, x.y);
        if (i == 3) break;
        x = tc::ffma2(from_e4m3x2(piece[i]), make_float2(-16.f, -16.f), tc::fmul2(x, make_float2(16.f, 16.f)));    // 16 (x - piece), exact
    }
}

// ---- pieces --------------------------------------------------------------------------------------
__device__ __forceinline__ int tiles_of(int rows) { return (rows + kTile - 1) / kTile; }

// How a call is cut; a warp finds it, each lane from some consecutive units.
struct Cut {
    int each, u0, u1;                    // this lane's units
    uint32_t mine, upto;                 // their tiles, of one head; with all units before
    uint32_t all, share;                 // tiles of all heads; of a block's piece, or 0:
    uint32_t per;                        // tiles of a range, or 0: blocks have one whole head or two
    uint32_t ranges, ranges_upto;        // ranges of a head of each of this lane's units; with all units before
    uint32_t sorted0, sorted1;           // whole heads, more than blocks: the units by falling length, those in places `lane` and 32 + lane: tiles * 64 + unit
};
constexpr int kMostSorted = 64;
// The tiles of the unit in place r, with its number, for a lane's own r.
__device__ __forceinline__ uint32_t sorted_unit(const Cut &c, uint32_t r) {
    const uint32_t a = __shfl_sync(0xFFFFFFFFu, c.sorted0, r & 31), b = __shfl_sync(0xFFFFFFFFu, c.sorted1, r & 31);
    return r < 32 ? a : b;
}
// Heads are not cut for a range kJoinTiles longer: joining costs that much.  With at most as many heads as blocks, ranges of a head each,
// unless they become kSwitchTiles longer than an even piece: the way from one head to the next costs where a block has few tiles (by ranges and by
// pieces: 12 sequences of up to 3000 rows, 4 heads, 14.0 and 15.5 us; 36 of 1690, 8 heads, 25.2 and 26.8; 4 of 2000, 12.8 and 13.5).  At most 64 ranges of a
// head, whose joining is the longer the more there are (one head of 33 792 rows by at most 16, 32 and 64 ranges, and by 132 pieces: 22.8, 17.4, 14.5 and
// 17.9 us; two heads 23.1, 17.9, 14.8, 15.6; eight 25.2, 23.5, 24.2, 23.6).
// With up to twice as many heads as blocks, of at most 64 units (two to a lane), a block has the i-th longest and the i-th last: 64 units of
// up to 1690 rows, 8 heads, 34.7 us so, 35.5 by pieces.  More units take pieces: 65 of 8 heads 36.6 us, 128 of 4 heads 35.5.
constexpr int kSwitchTiles = 4, kMostRanges = 64;
__device__ __forceinline__ Cut make_cut(const AttnArgs &A) {
    Cut c;
    const int lane = lane_id();
    c.each = (A.U + 31) >> 5;
    c.u0 = min(A.U, lane * c.each);
    c.u1 = min(A.U, c.u0 + c.each);
    c.mine = 0;
    int longest = 0;
#pragma unroll 4
    for (int u = c.u0; u < c.u1; ++u) {
        const int t = tiles_of(unit_rows(A, u));
        c.mine += t;
        longest = max(longest, t);
    }
    c.upto = c.mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, c.upto, o);
        if (lane >= o) c.upto += x;
        longest = max(longest, __shfl_xor_sync(0xFFFFFFFFu, longest, o));
    }
    const uint32_t blocks = gridDim.x, heads = (uint32_t)A.U * A.Hkv;
    c.all = __shfl_sync(0xFFFFFFFFu, c.upto, 31) * A.Hkv;
    c.share = (c.all + blocks - 1) / blocks;
    c.sorted0 = c.sorted1 = 0;
    c.per = c.ranges = c.ranges_upto = 0;
    const uint32_t most = c.share + kJoinTiles;
    if (heads <= blocks) {
        auto count = [&](uint32_t per) {                              // ranges of a head of each unit, by lane
            uint32_t n = 0;
#pragma unroll 2
            for (int u = c.u0; u < c.u1; ++u) n += ((uint32_t)tiles_of(unit_rows(A, u)) + per - 1) / per;
            return n;
        };
        const uint32_t least = max(max(1u, c.share), (uint32_t)(longest + kMostRanges - 1) / kMostRanges);
        for (uint32_t per = least; per <= least + kSwitchTiles || per + kJoinTiles >= (uint32_t)longest; ++per) {
            if (per + kJoinTiles >= (uint32_t)longest) per = max(1, longest);
            c.ranges = count(per);
            if (__reduce_add_sync(0xFFFFFFFFu, c.ranges) * A.Hkv > blocks) continue;
            c.ranges_upto = c.ranges;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, c.ranges_upto, o);
                if (lane >= o) c.ranges_upto += x;
            }
            c.per = per;
            c.share = 0;
            break;
        }
        return c;
    }
    if (heads > 2 * blocks || A.U > kMostSorted || longest > most) return c;
    {
        // units by length: a unit's place is the number of longer ones, or as long ones before it
        uint32_t mine[2], place[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = lane + 32 * i;
            mine[i] = u < A.U ? (uint32_t)tiles_of(unit_rows(A, u)) * 64 + 63 - u : 0;       // (all different, and 0 for none)
        }
        for (int k = 0; k < 32; ++k) {
            const uint32_t a = __shfl_sync(0xFFFFFFFFu, mine[0], k), b = __shfl_sync(0xFFFFFFFFu, mine[1], k);
#pragma unroll
            for (int i = 0; i < 2; ++i) place[i] += (a > mine[i]) + (b > mine[i]);
        }
        for (int k = 0; k < 32; ++k) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t at = __shfl_sync(0xFFFFFFFFu, place[i], k), is = __shfl_sync(0xFFFFFFFFu, mine[i], k) ^ 63;      // (63 - u back to u)
                if (k + 32 * i < A.U) {
                    if (at == (uint32_t)lane) c.sorted0 = is;
                    if (at == (uint32_t)lane + 32) c.sorted1 = is;
                }
            }
        }
        // the longest pair: of each unit's heads the last one that comes first in a block, since it has the longest partner
        uint32_t pair = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = lane + 32 * i, item = min(r * A.Hkv + A.Hkv - 1, blocks - 1), partner = 2 * blocks - 1 - item;
            const uint32_t with = sorted_unit(c, partner < heads ? partner / A.Hkv : 0) >> 6;
            if (r < (uint32_t)A.U && r * A.Hkv < blocks) pair = max(pair, ((i ? c.sorted1 : c.sorted0) >> 6) + (partner < heads ? with : 0));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) pair = max(pair, __shfl_xor_sync(0xFFFFFFFFu, pair, o));
        if (pair > most) return c;
    }
    c.share = 0;
    return c;
}

// Tiles [t0, t1) of the head (u, h), whose first tile has the number `head`; t0 has the number x, the piece goes to `end`.
struct Walk { int u, h, rows, tiles, t0, t1; uint32_t x, end, head; };

// Where tile x is; x below c.all.  Called by a whole warp.
__device__ __forceinline__ void walk_to(const AttnArgs &A, const Cut &c, uint32_t x, uint32_t end, Walk &w) {
    const uint32_t H = A.Hkv;
    const int owner = __ffs(__ballot_sync(0xFFFFFFFFu, x < c.upto * H)) - 1;
    int u = 0;
    uint32_t base = 0;                                                // tiles of a head of each of the units before
    if (lane_id() == owner) {
        base = c.upto - c.mine;
        for (u = c.u0; u < c.u1 - 1; ++u) {
            const int t = tiles_of(unit_rows(A, u));
            if (x < (base + t) * H) break;
            base += t;
        }
    }
    w.u = __shfl_sync(0xFFFFFFFFu, u, owner);
    base = __shfl_sync(0xFFFFFFFFu, base, owner) * H;
    w.rows = unit_rows(A, w.u);
    w.tiles = tiles_of(w.rows);
    w.h = (x - base) / (uint32_t)w.tiles;
    w.head = base + w.h * w.tiles;
    w.t0 = x - w.head;
    w.x = x;
    w.end = end;
    w.t1 = min(w.tiles, w.t0 + (int)(end - x));
}
// The block's range; false where there is none.  Ranges are numbered by unit, head and key.
__device__ __forceinline__ bool walk_range(const AttnArgs &A, const Cut &c, Walk &w) {
    const uint32_t H = A.Hkv, i = blockIdx.x, hit = __ballot_sync(0xFFFFFFFFu, i < c.ranges_upto * H);
    if (hit == 0) return false;
    const int owner = __ffs(hit) - 1;
    int u = 0;
    uint32_t base = 0, n = 0;                                         // ranges of all heads of the units before; of one of this unit's
    if (lane_id() == owner) {
        base = (c.ranges_upto - c.ranges) * H;
        for (u = c.u0; u < c.u1; ++u) {
            n = ((uint32_t)tiles_of(unit_rows(A, u)) + c.per - 1) / c.per;
            if (i < base + n * H) break;
            base += n * H;
        }
    }
    w.u = __shfl_sync(0xFFFFFFFFu, u, owner);
    n = __shfl_sync(0xFFFFFFFFu, n, owner);
    const uint32_t in = i - __shfl_sync(0xFFFFFFFFu, base, owner);
    w.h = in / n;
    w.rows = unit_rows(A, w.u);
    w.tiles = tiles_of(w.rows);
    w.t0 = (in - w.h * n) * c.per;
    w.t1 = min(w.tiles, w.t0 + (int)c.per);
    w.x = w.head = 0;
    w.end = w.t1 - w.t0;
    return true;
}
// Whole heads: the block's first or second one.
__device__ __forceinline__ bool walk_head(const AttnArgs &A, const Cut &c, int second, Walk &w) {
    const uint32_t blocks = gridDim.x, heads = (uint32_t)A.U * A.Hkv, i = second ? 2 * blocks - 1 - blockIdx.x : blockIdx.x;
    if (i >= heads) return false;
    const uint32_t r = i / A.Hkv;
    w.u = heads <= blocks ? r : sorted_unit(c, r) & 63;
    w.h = i - r * A.Hkv;
    w.rows = unit_rows(A, w.u);
    w.tiles = w.t1 = tiles_of(w.rows);
    w.t0 = 0;
    w.x = w.head = 0;
    w.end = w.tiles;
    return w.tiles > 0;
}
// The block's piece; false where there is none.
__device__ __forceinline__ bool walk_piece(const AttnArgs &A, const Cut &c, Walk &w) {
    if (c.share == 0) return c.per != 0 ? walk_range(A, c, w) : walk_head(A, c, 0, w);
    const uint32_t x = blockIdx.x * c.share;
    if (x >= c.all) return false;
    walk_to(A, c, x, min(c.all, x + c.share), w);
    return true;
}
// On to the next head of the piece; false at its end.
__device__ __forceinline__ bool walk_next(const AttnArgs &A, Walk &w) {
    w.x += w.t1 - w.t0;
    if (w.x >= w.end) return false;
    if (++w.h == A.Hkv) {
        w.h = 0;
        do { ++w.u; w.rows = unit_rows(A, w.u); w.tiles = tiles_of(w.rows); } while (w.tiles == 0 && w.u < A.U - 1);
    }
    w.head = w.x;
    w.t0 = 0;
    w.t1 = min(w.tiles, (int)(w.end - w.x));
    return true;
}

// What a group is, from the loader to the other warps.
struct Task {
    int n, t, rows, u, h;                // tiles (0: no more groups), the first one's place in the unit, the unit's rows, unit, head
    int record;                          // where the part of the head goes: -1: it is all of it, else the record's number
    int place;                           // 1: first, 2: last of the head's groups in the piece
    int next;                            // the first query row of the next head in the block, or -1
};
static_assert(sizeof(Task) == 32, "as much as Lay::kSmemTask leaves");

// A lane's part of a query, two or four elements.
template <int D> struct alignas(D / 16) Query { uint32_t w[D / 64]; };
// A query head's rows of the operand, by a warp.  Rows by half, piece, head.  Returns the factor of its logits:
// the queries' power of two and the softmax's scale; NaN for a query that is not finite.
template <int D>
__device__ __forceinline__ float put_query(uint32_t operand, int g, const Query<D> &v, float scale_log2) {
    constexpr int V = D / 32;
    const int lane = lane_id();
    float x[V];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) { x[2 * i] = __uint_as_float(v.w[i] << 16); x[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u); }
    float size = 0.f;
    bool fine = true;
#pragma unroll
    for (int i = 0; i < V; ++i) { size = fmaxf(size, fabsf(x[i])); fine = fine && is_finite(x[i]); }
    if (!fine) size = __uint_as_float(0x7F800000u);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) size = fmaxf(size, __shfl_xor_sync(0xFFFFFFFFu, size, o));
    const int ex = is_finite(size) ? max(-100, (int)(__float_as_uint(size) >> 23) - 127) - 7 : 0;   // the largest element to [128, 256)
    const float f = power_of_two(-ex);
    uint32_t lo[V / 2], hi[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float a = x[2 * i] * f, b = x[2 * i + 1] * f;
        hi[i] = to_e4m3x2(a, b);
        const float2 h = from_e4m3x2(hi[i]);
        lo[i] = to_e4m3x2((a - h.x) * 16.f, (b - h.y) * 16.f);
    }
    const int n = (g >> 2) * 8 + (g & 3), c = lane * V >> 4;
    const uint32_t at = operand + (lane * V & 15), first = at + Lay<D>::chunk(n, c), second = at + Lay<D>::chunk(n + 4, c);
    if constexpr (V == 4) {
        sts32(first, hi[0] | hi[V / 2 - 1] << 16);
        sts32(second, lo[0] | lo[V / 2 - 1] << 16);
    } else {
        sts16(first, hi[0]);
        sts16(second, lo[0]);
    }
    return is_finite(size) ? power_of_two(ex) * scale_log2 : __uint_as_float(0x7FC00000u);
}

// kByTiles: at most four query heads, or two (kPairs: of one half), the halves take every other tile; else the halves have four heads each.
template <int D, bool kByTiles, int kPairs>
__global__ void __launch_bounds__(kThreads, 2)
cache_attention_tc_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttnArgs A) {
    typedef Lay<D> L;
    constexpr int kStages = L::kStages, kHeads = kByTiles ? kHalf : kMaxHeads;       // heads served
    constexpr int kShift = D == 128 ? 7 : 6;                         // bytes of a row, as a shift
    extern __shared__ __align__(1024) uint8_t ptc_smem[];
    const uint32_t base = tc::smem_u32(ptc_smem), bars = base + L::kSmemBar;
    const int warp = tc::warp_number(), lane = threadIdx.x & 31;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(ptc_smem + L::kSmemBar + 8 * L::kNumBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *cta_status = reinterpret_cast<int *>(tmem_slot + 2);
    float *info = reinterpret_cast<float *>(ptc_smem + L::kSmemInfo), *factors = reinterpret_cast<float *>(ptc_smem + L::kSmemFactor);
    if ((base & 1023u) != 0) {                       // the swizzled tiles need a 1024-byte aligned base
        predecessor_done();
        if (threadIdx.x == 0) {
            report(A.status, 6);
            if (A.cut_heads) A.cut_heads[blockIdx.x] = make_int4(0, 0, 0, 0);
        }
        return;
    }
    auto bar = [&](int i) { return bars + 8u * i; };
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kNumBars; ++i)
            tc::mbar_init(bar(i), i == L::kBarPFull || i == L::kBarPFull + 1 ? (kByTiles ? 128 : 256) : i >= L::kBarIEmpty ? 257
                                  : i == L::kBarQFull || i == L::kBarQFull + 1 ? kHeads : 1);
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

    const int G = A.G, tile_pages = kTile >> A.page_shift, record = record_floats(G, D);
    auto query = [&](int first, int g) {                             // of a head's first query row and a number
        return g < G ? *reinterpret_cast<const Query<D> *>(static_cast<const __nv_bfloat16 *>(A.q) + ((int64_t)first + g) * D + lane * (D / 32)) : Query<D>{};
    };
    Task *tasks = reinterpret_cast<Task *>(ptc_smem + L::kSmemTask);
    // the next group's task, for the warps that do the loader's bidding
    auto wait_task = [&](int group, Task &t) {
        if (!tc::mbar_wait_warp(bar(L::kBarTask + group % kInfos), group / kInfos & 1, abort_flag, cta_status)) return false;
        t = tasks[group % kInfos];
        return t.n != 0;
    };
    if (warp == 0) {
        // A group's pages, two a lane: their numbers, and their scales.
        struct Pages { int a, b; float ka, kb, va, vb; };
        auto numbers = [&](const Task &g, Pages &p) {
            const int j = (g.t << (7 - A.page_shift)) + lane, end = min((g.rows + A.page - 1) >> A.page_shift, (g.t + g.n) << (7 - A.page_shift));
            const int *table = A.table + (int64_t)g.u * A.max_pages;
            p.a = j < end ? table[j] : 0;
            p.b = j + 32 < end ? table[j + 32] : 0;
            if ((unsigned)p.a >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); p.a = 0; }
            if ((unsigned)p.b >= (unsigned)A.n_pages) { report(A.status, kStatusIndex); p.b = 0; }
        };
        auto scales = [&](int h, Pages &p) {
            const int64_t a = (int64_t)p.a * A.Hkv + h, b = (int64_t)p.b * A.Hkv + h;
            p.ka = A.k_scale[a]; p.va = A.v_scale[a];
            if (lane + 32 < kGroup * tile_pages) { p.kb = A.k_scale[b]; p.vb = A.v_scale[b]; }
        };
        int st = 0, phase = 0;
        struct Group { Task is; Pages p; };
        auto load_tile = [&](const CUtensorMap *m, const Group &g, int i) {
            if (!tc::mbar_wait_warp(bar(L::kBarEmpty + st), phase ^ 1, abort_flag, cta_status)) return false;
            const int slot = i * tile_pages + lane;
            const int x = __shfl_sync(0xFFFFFFFFu, g.p.a, slot & 31), y = __shfl_sync(0xFFFFFFFFu, g.p.b, slot & 31), id = slot < 32 ? x : y;
            const int here = min(tile_pages, ((g.is.rows + A.page - 1) >> A.page_shift) - (g.is.t + i) * tile_pages);     // pages of the tile that there are
            if (tc::elect_one()) tc::mbar_expect_tx(bar(L::kBarFull + st), (uint32_t)here << (A.page_shift + kShift));
            __syncwarp();
            if (lane < here) tc::tma_load_4d(base + st * L::kStageBytes + ((uint32_t)lane << (A.page_shift + kShift)), m, bar(L::kBarFull + st), 0, 0, g.is.h, id);
            __syncwarp();
            if (++st == kStages) { st = 0; phase ^= 1; }
            return true;
        };
        auto load_tiles = [&](const Group &k, const Group &v) {
            bool ok = true;
            for (int i = 0; ok && i < max(k.is.n, v.is.n); ++i) {
                if (i < k.is.n) ok = load_tile(&kmap, k, i);
                if (ok && i < v.is.n) ok = load_tile(&vmap, v, i);
            }
            return ok;
        };
        // (a call whose heads cannot be cut has one for each block at most: nothing to find)
        Cut cut = {};
        if (A.cut_heads) cut = make_cut(A);
        Walk w = {}, ahead = {};                                     // the head of the group after `now`, and the one after it
        int group = 0, second = 0;
        int4 cut_head = make_int4(0, 0, 0, 0);                       // a head that begins here and goes on in other blocks
        bool more = walk_piece(A, cut, w), more_ahead = false;
        auto look_ahead = [&]() {
            ahead = w;
            more_ahead = walk_next(A, ahead);
            if (!more_ahead && cut.share == 0 && !second) more_ahead = walk_head(A, cut, second = 1, ahead);
        };
        auto set = [&](Group &g, int t) {
            g.is.n = min(kGroup, w.t1 - t); g.is.t = t; g.is.rows = w.rows; g.is.u = w.u; g.is.h = w.h;
            g.is.place = (t == w.t0 ? 1 : 0) | (t + g.is.n == w.t1 ? 2 : 0);
            g.is.next = more_ahead ? ahead.u * A.Hq + ahead.h * G : -1;
            g.is.record = w.t0 == 0 && w.t1 == w.tiles ? -1 : 2 * (int)blockIdx.x + (w.t0 == 0);
            if (w.t0 == 0 && w.t1 < w.tiles) cut_head = make_int4(w.u, w.h * G,
                cut.share == 0 ? (w.tiles + (int)cut.per - 1) / (int)cut.per : (int)((w.head + w.tiles - 1) / cut.share - blockIdx.x + 1), G);
            numbers(g.is, g.p);
        };
        bool ok = true;
        Group now, next, before;
        now.is.n = before.is.n = 0;
        if (more) {
            if (A.cut_heads && cut.per == 0) look_ahead();           // (a range is the block's only one)
            set(now, w.t0);
            scales(now.is.h, now.p);
        }
        while (true) {
            // the task, K's tiles with those of V of the group before, the scales
            const int buffer = group % kInfos;
            ok = tc::mbar_wait_warp(bar(L::kBarIEmpty + buffer), (group / kInfos & 1) ^ 1, abort_flag, cta_status);
            if (!ok) break;
            if (lane == 0) {
                tasks[buffer] = now.is;
                tc::mbar_arrive(bar(L::kBarTask + buffer));
            }
            if (now.is.n == 0) break;
            // the group after this one: its pages' numbers on their way
            next.is.n = 0;
            if (!(now.is.place & 2)) {
                set(next, now.is.t + now.is.n);
            } else if (more_ahead) {
                w = ahead;
                look_ahead();
                set(next, w.t0);
            }
            ok = load_tiles(now, before);
            if (!ok) break;
            float *to = info + buffer * kInfo;
            to[lane] = now.p.ka; to[kMostPages + lane] = log2_of(now.p.va);
            if (lane + 32 < kMostPages) { to[lane + 32] = now.p.kb; to[kMostPages + lane + 32] = log2_of(now.p.vb); }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar(L::kBarIFull + buffer));
            if (next.is.n != 0) scales(next.is.h, next.p);
            before = now; now = next; ++group;
        }
        if (A.cut_heads && lane == 0) A.cut_heads[blockIdx.x] = cut_head;
        if (ok) ok = load_tiles(now, before);                        // (no tiles of K: the last group's V)
        tc::copies_land(bar(L::kBarFull), 8, kStages, st, phase);
    } else if (warp == 1) {
        int st = 0, phase = 0, tile = 0, made = 0;                   // made: the logits' bars, in turn
        auto next = [&]() { if (++st == kStages) { st = 0; phase ^= 1; } };
        auto logits = [&](int group, int t, uint32_t q_lo) {
            if (!tc::mbar_wait_warp(bar(L::kBarFull + st), phase, abort_flag, cta_status)) return false;
            tc::tc_fence_after();
            const uint32_t a_lo = tc::desc_lo(base + st * L::kStageBytes), at = tmem + kColS + ((group & 1) * kGroup + t) * kQCols;
            if (tc::elect_one()) {
#pragma unroll
                for (int j = 0; j < D / 32; ++j) umma_e4m3(at, a_lo + 2 * j, L::kDescHi, q_lo + 2 * j, L::kDescHi, kIdescQK, j > 0);
                tc::umma_commit(bar(L::kBarEmpty + st));
                tc::umma_commit(bar(L::kBarS + made));
            }
            __syncwarp();
            if (++made == 2 * kGroup) made = 0;
            next();
            return true;
        };
        auto output = [&](int t, int n, int valid) {                 // valid: rows of the last tile that the unit has
            const int pb = tile & 1;
            if (!tc::mbar_wait_warp(bar(L::kBarFull + st), phase, abort_flag, cta_status)) return false;
            if (t == n - 1 && valid < kTile) {
                // rows of V behind the unit's last one: zeros, since a weight of zero times a NaN would not be nothing
                for (int i = valid * (D / 16) + lane; i < kTile * (D / 16); i += 32) tc::sts128(base + st * L::kStageBytes + i * 16, 0.f, 0.f, 0.f, 0.f);
                fence_proxy_async();
                __syncwarp();
            }
            if (!tc::mbar_wait_warp(bar(L::kBarPFull + pb), (tile >> 1) & 1, abort_flag, cta_status)) return false;
            tc::tc_fence_after();
            const uint32_t a_lo = tc::desc_lo(base + st * L::kStageBytes), p_lo = tc::desc_lo(base + L::kSmemP + pb * kPBytes);
            if (tc::elect_one()) {
#pragma unroll
                for (int j = 0; j < 4; ++j) umma_e4m3(tmem, a_lo + 2 * D * j, L::kDescHi, p_lo + 64 * j, kDescPHi, kIdescPV, (t | j) != 0);
                tc::umma_commit(bar(L::kBarEmpty + st));
                tc::umma_commit(bar(L::kBarPEmpty + pb));
                if (t == n - 1) tc::umma_commit(bar(L::kBarO));
            }
            __syncwarp();
            ++tile;
            next();
            return true;
        };
        Task now;
        bool ok = true;
        int group = 0, head = -1, before_n = 0, before_valid = 0;
        uint32_t q_lo = 0;
        while (wait_task(group, now)) {
            if (tc::elect_one()) tc::mbar_arrive(bar(L::kBarIEmpty + group % kInfos));
            __syncwarp();
            if (now.place & 1) {
                ++head;
                q_lo = tc::desc_lo(base + L::kSmemQ + (head & 1) * L::kQBytes);
                ok = tc::mbar_wait_warp(bar(L::kBarQFull + (head & 1)), head >> 1 & 1, abort_flag, cta_status);
            }
            for (int i = 0; ok && i < max(now.n, before_n); ++i) {   // (as the loader sends them)
                if (i < now.n) ok = logits(group, i, q_lo);
                if (ok && i < before_n) ok = output(i, before_n, before_valid);
            }
            if (!ok) break;
            before_n = now.n;
            before_valid = min(kTile, now.rows - (now.t + now.n - 1) * kTile);
            ++group;
        }
        for (int i = 0; ok && i < before_n; ++i) ok = output(i, before_n, before_valid);
    } else {
        const int e = threadIdx.x - 64, half = e >> 7;               // 0 .. 255
        const int row = 32 * (warp & 3) + lane;                      // TMEM lane this thread reads: key of a tile / output dim
        const uint32_t trow = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const int set = kByTiles ? 0 : half, g0 = kHalf * set;       // this half's heads
        constexpr int parts = kByTiles ? 2 : 1;                      // ... and tiles: all, or those with the number of the half
        const uint32_t tcols = trow + set * 8;                       // columns of their logits within a tile's
        float *red = reinterpret_cast<float *>(ptc_smem + L::kSmemRed);
        Task now = {}, done = {};
        Query<D> q = {};
        const int own = (int)blockIdx.x * G;                         // a call whose heads cannot be cut: the block's head is known before the lengths are
        if (!A.cut_heads && own < A.U * A.Hq) q = query(own, e >> 5);
        // a head's operand, a warp per query head; with the number of the head in the block
        auto put = [&](int head) {
            if ((e >> 5) >= kHeads) return;
            const float f = put_query<D>(base + L::kSmemQ + (head & 1) * L::kQBytes, e >> 5, q, A.scale_log2);
            if (lane == 0) factors[(head & 1) * kMaxHeads + (e >> 5)] = f;
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar(L::kBarQFull + (head & 1)));
        };
        // The group's task; false behind the last one.  A warp whose wait has run out goes on, without work, to the next meeting: they are
        // as many for every warp.
        bool ok = true;
        auto take_task = [&](int group) {
            ok = ok && tc::mbar_wait_warp(bar(L::kBarTask + group % kInfos), group / kInfos & 1, abort_flag, cta_status);
            if (ok) now = tasks[group % kInfos];
            return !ok || now.n != 0;
        };
        bool more = take_task(0);
        if (ok && more) {
            if (A.cut_heads) q = query(now.u * A.Hq + now.h * G, e >> 5);
            put(0);
        }
        bool together = epi_all(ok);

        float cq[kHalf], m[kHalf], mr[kHalf], l[kHalf], acc[kHalf];  // m: the maximum; mr: of the weights with V's scales, above it
        auto add_output = [&](int group) {                           // a group's product into acc
            if (kByTiles && half != 0) return;                       // (one thread a dim is enough)
            ok = ok && tc::mbar_wait_warp(bar(L::kBarO), group & 1, abort_flag, cta_status);
            if (!ok) return;
            tc::tc_fence_after();
            float o[8], o2[8];
            tmem_ld8(trow + set * 16, o);
            tmem_ld8(trow + set * 16 + 8, o2);
            tmem_ld_wait(o);
            tmem_ld_wait(o2);
#pragma unroll
            for (int g = 0; g < kHalf; ++g) acc[g] += fmaf(fmaf(fmaf(o2[4 + g], 0.0625f, o2[g]), 0.0625f, o[4 + g]), 0.0625f, o[g]);
        };
        // A head is finished behind the barrier of the group after it: its sums of weights have been left in `all` before.
        auto leave_sums = [&](float *all) {
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                const float sum = warp_sum(l[g]);
                if (lane == 0) all[(e >> 5) * 3 * kHalf + 2 * kHalf + g] = sum;
            }
        };
        auto finish = [&](const Task &t, const float *all) {
            if ((kByTiles && half != 0) || row >= D || !ok) return;
            float *out = A.out + ((int64_t)t.u * A.Hq + t.h * G) * D + row, *part = A.part + (int64_t)t.record * record;
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                if (g0 + g < G) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4 * parts; ++i) sum += all[(4 * (kByTiles ? 0 : half) + i) * 3 * kHalf + 2 * kHalf + g];
                    const float o = acc[g] * tc::ex2(mr[g] - 8.f);       // relative to the logits' maximum
                    if (t.record < 0) {
                        out[(g0 + g) * D] = o / sum;
                    } else {
                        part[(g0 + g) * D + row] = o;
                        if (row == 0) { part[G * D + g0 + g] = m[g]; part[G * D + G + g0 + g] = sum; }
                    }
                }
            }
        };
        int group = 0, head = -1, tile = 0;
        for (; together && more; ++group, more = take_task(group)) {
            const int n = now.n, first_key = now.t * kTile, buffer = group % kInfos;
            const int from = kByTiles ? (tile + half) & 1 : 0;       // this half's first tile of the group
            const bool first = now.place & 1;
            head += first;
            const float *in = info + buffer * kInfo;
            if (first && now.next >= 0) q = query(now.next, e >> 5); // (on its way)
            ok = ok && tc::mbar_wait_warp(bar(L::kBarIFull + buffer), group / kInfos & 1, abort_flag, cta_status);
            float top[kHalf], topv[kHalf];
#pragma unroll
            for (int g = 0; g < kHalf; ++g) { top[g] = kLowest; topv[g] = kLowest; }
            const uint32_t scol = tcols + kColS + (group & 1) * kGroup * kQCols;
            float s[8];
            // The logits are there one after the other: of the first group each is waited for, of the others, which have been
            // made beside the group before, the last one.
            auto wait_logits = [&](int t) {
                const int turn = (tile + t) / (2 * kGroup);
                ok = ok && tc::mbar_wait_warp(bar(L::kBarS + tile + t - turn * 2 * kGroup), turn & 1, abort_flag, cta_status);
                tc::tc_fence_after();
            };
            if (group > 0 && from < n) wait_logits(n - 1);
            // (a head's factors are there when its logits are, the first one's from the beginning)
#pragma unroll
            for (int g = 0; g < kHalf; ++g) cq[g] = factors[(head & 1) * kMaxHeads + g0 + g];
            if (ok && group > 0 && from < n) tmem_ld8(scol + from * kQCols, s);
            for (int t = from; t < n; t += parts) {
                if (group == 0) {
                    wait_logits(t);
                    if (ok) tmem_ld8(scol + t * kQCols, s);
                }
                tmem_ld_wait(s);                                     // (also where a wait has run out with a read on its way)
                if (!ok) continue;
                float z[kHalf];
#pragma unroll
                for (int g = 0; g < kHalf; ++g) z[g] = fmaf(s[4 + g], 0.0625f, s[g]);
                if (group > 0 && t + parts < n) tmem_ld8(scol + (t + parts) * kQCols, s);
                if (first_key + t * kTile + row < now.rows) {
                    const int j = (t * kTile + row) >> A.page_shift;
                    const float ks = in[j], lv = in[kMostPages + j];
#pragma unroll
                    for (int g = 0; g < kHalf; ++g) {
                        const float x = __fmul_rn(z[g], ks * cq[g]);
                        top[g] = fmaxf(top[g], x);
                        topv[g] = fmaxf(topv[g], x + lv);
                    }
                }
            }
            float *all = red + (group & 1) * 8 * 3 * kHalf;
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                top[g] = warp_max(top[g]);
                topv[g] = warp_max(topv[g]);
                if (lane == 0) { all[(e >> 5) * 3 * kHalf + g] = top[g]; all[(e >> 5) * 3 * kHalf + kHalf + g] = topv[g]; }
            }
            if (group > 0) {                                     // (before the barrier: behind it this group's product may begin)
                add_output(group - 1);
                tc::tc_fence_before();
                if (first) leave_sums(all);
            }
            if (!epi_all(ok)) {
                together = false;
                break;
            }
            if (first) {
                if (group > 0) finish(done, all);
                // (the logits of the head before this one are made, and every thread has done with its factors)
                if (now.next >= 0) put(head + 1);
#pragma unroll
                for (int g = 0; g < kHalf; ++g) { m[g] = kLowest; mr[g] = 0.f; l[g] = 0.f; acc[g] = 0.f; }
                done = now;
            }
            // Beyond kFar log2 of V's scale is lost next to a logit, and the difference of the two maxima is not what it should be: the second one is
            // then said to be the largest of the group's scales above the first, which no weight passes either.  (Found in every group: under a branch for the
            // far ones the code around it was slower, 72.8 us for 71.2, 200 units of up to 2200 rows, 8 heads of 4 query heads of 64.)
            float a[kHalf], b[kHalf];
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                a[g] = m[g]; b[g] = kLowest;
#pragma unroll
                for (int i = 0; i < 4 * parts; ++i) {
                    const float *of = all + (4 * (kByTiles ? 0 : half) + i) * 3 * kHalf;
                    a[g] = fmaxf(a[g], of[g]);
                    b[g] = fmaxf(b[g], of[kHalf + g]);
                }
            }
            const int pages = (min(n * kTile, now.rows - first_key) + A.page - 1) >> A.page_shift;
            const float most = warp_max(fmaxf(lane < pages ? in[kMostPages + lane] : kLowest, lane + 32 < pages ? in[kMostPages + lane + 32] : kLowest));
#pragma unroll
            for (int g = 0; g < kHalf; ++g) {
                const float up = m[g] - a[g], r = fmaxf(mr[g] + up, fabsf(a[g]) > kFar ? most : b[g] - a[g]);
                l[g] *= tc::ex2(up);
                acc[g] *= tc::ex2(up + (mr[g] - r));
                m[g] = a[g]; mr[g] = r;
            }
            if (ok && from < n) tmem_ld8(scol + from * kQCols, s);
            for (int t = from; t < n; t += parts) {
                const int i = tile + t, pb = i & 1;
                tmem_ld_wait(s);
                if (!ok) continue;
                const bool valid = first_key + t * kTile + row < now.rows;
                const int j = (t * kTile + row) >> A.page_shift;
                const float ks = in[j], lv = in[kMostPages + j] + 8.f;                  // (weights times 256)
                float2 x[kPairs];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    // two heads at once; but for the products, which are rounded as for the maximum, so that none is above it: two at once were
                    // compiled into one step with the difference, without a rounding between
                    const int g = 2 * i;
                    const float2 z = tc::ffma2(make_float2(s[4 + g], s[5 + g]), make_float2(0.0625f, 0.0625f), make_float2(s[g], s[g + 1]));
                    const float2 c = tc::fmul2(make_float2(ks, ks), make_float2(cq[g], cq[g + 1]));
                    const float2 d = tc::fadd2(make_float2(__fmul_rn(z.x, c.x), __fmul_rn(z.y, c.y)), make_float2(-m[g], -m[g + 1]));
                    const float2 dv = tc::fadd2(d, tc::fadd2(make_float2(lv, lv), make_float2(-mr[g], -mr[g + 1])));
                    l[g] += valid ? tc::ex2(d.x) : 0.f;
                    l[g + 1] += valid ? tc::ex2(d.y) : 0.f;
                    x[i].x = valid ? tc::ex2(dv.x) : 0.f;
                    x[i].y = valid ? tc::ex2(dv.y) : 0.f;
                }
                if (t + parts < n) tmem_ld8(scol + (t + parts) * kQCols, s);
                uint32_t lower[4], word[4];
                four_pieces(x[0], lower);
                if constexpr (kPairs == 2) {
                    four_pieces(x[kPairs - 1], word);
#pragma unroll
                    for (int k = 0; k < 4; ++k) word[k] = lower[k] | word[k] << 16;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) word[k] = lower[k];
                }
                ok = tc::mbar_wait_warp(bar(L::kBarPEmpty + pb), ((i >> 1) & 1) ^ 1, abort_flag, cta_status);
                if (!ok) continue;
                // the key's row of the operand: 32 weights by half, piece, head; the swizzle exchanges the halves of every other four rows
                sts128(base + L::kSmemP + pb * kPBytes + row * 32 + ((set ^ ((row >> 2) & 1)) << 4), word);
                fence_proxy_async();
                tc::tc_fence_before();
                tc::mbar_arrive(bar(L::kBarPFull + pb));
            }
            tc::mbar_arrive(bar(L::kBarIEmpty + buffer));
            tile += n;
        }
        if (together && group > 0) {
            add_output(group - 1);
            float *all = red + (group & 1) * 8 * 3 * kHalf;
            leave_sums(all);
            if (epi_all(ok)) finish(done, all);
        }
    }
    // units without rows, shared out over the blocks
    for (int u = blockIdx.x; u < A.U; u += gridDim.x) {
        const int n = A.rows[u];
        if (n < 0 || n > A.max_pages << A.page_shift) { if (threadIdx.x == 0) report(A.status, kStatusIndex); }
        if (n <= 0)
            for (int i = threadIdx.x; i < A.Hq * D; i += kThreads) A.out[(int64_t)u * A.Hq * D + i] = 0.f;
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 1) tc::tmem_dealloc(tmem, kTmemCols);
    if (threadIdx.x == 0 && *abort_flag != 0) report(A.status, *cta_status);
}

}  // namespace ptc
}  // namespace paged
}  // namespace flowmm
