// Sequences packed one behind the other, each attending to its own earlier tokens: what the forward and the backward kernels share.
//
// The buffer's tokens fall into segments: those in front of the first sequence, the sequences, those behind the last.  A workgroup has a
// tile of one segment, `size` rows that begin with the segment's.  Tile t of a segment that begins with row r (of all rows of a key head)
// and is number i has place floor(r / size) + i + t: the segments' places do not overlap (floor(x + y) >= floor(x) + floor(y)), there are
// at most floor(rows / size) + segments of them, and so the host, which does not know the lengths, knows how many workgroups it takes, and
// nothing needs a sum over the lengths or a launch in front.
//
// Which tile a workgroup has: of 64 segments, whose places are those of their first one on, the tiles with the longest walks first, found
// by a search for the length that as many tiles have as there are workgroups in front (24 sequences of 60 to 1,000 tokens, 12 heads of 64:
// 21.7 us in the place of 25.6 with the places' order).
#ifndef GRKAN_PACKED_H_
#define GRKAN_PACKED_H_

#include "grkan_attention.h"

namespace grkan {
namespace attention {

struct Packed : Args { // rows: of all tokens; batch and the operands' batch strides: not used
    char *rest; // what the rounding of `out` left, or null
    const void *offsets;
    int32_t offsets_64, sequences;
    int32_t tokens, each; // each: of a sequence, where there are no offsets
    int32_t slots;        // places, and so workgroups, of a key head
    int32_t value_tiles;  // places of tiles of 128 keys, whose values' lengths are kept
    int32_t parts, slab;  // keys' gradients: over how many workgroups the rows of a tile of keys are split at most, and tiles of rows of each
};

// Where segment i begins: i = 0 .. sequences + 2, the last being the end.
__device__ __forceinline__ int32_t boundary(const Packed &a, int32_t i)
{
    if (i <= 0)
        return 0;
    if (i >= a.sequences + 2)
        return a.tokens;
    if (!a.offsets)
        return (i - 1) * a.each;
    const int64_t n = a.offsets_64 ? static_cast<const int64_t *>(a.offsets)[i - 1] : (int64_t) static_cast<const int32_t *>(a.offsets)[i - 1];
    return (int32_t)(n < 0 ? 0 : n < a.tokens ? n : a.tokens);
}

struct Segment {
    int32_t first, count; // tokens
    int32_t tile;
    int32_t index;
    bool none; // of no sequence
};

// unit: rows of a token.  Offsets that fall give tiles within the buffer, but there may be more of them than places: some are nobody's then, of any segment.
template <int SIZE> __device__ __forceinline__ int32_t place_of(int32_t token, int32_t unit, int32_t i)
{
    return (int32_t)((uint32_t)token * (uint32_t)unit / (uint32_t)SIZE) + i;
}

// The wavefront's numbers, none of them negative, put together.
template <class Op> __device__ __forceinline__ int32_t of_lanes(int32_t v, Op &&op)
{
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true));
    const auto rows = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = op((int32_t)rows[0], (int32_t)rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    return __builtin_amdgcn_readfirstlane(op((int32_t)halves[0], (int32_t)halves[1]));
}
__device__ __forceinline__ int32_t sum_of_lanes(int32_t v)
{
    return of_lanes(v, [](int32_t x, int32_t y) { return x + y; });
}
__device__ __forceinline__ int32_t largest_of_lanes(int32_t v)
{
    return of_lanes(v, [](int32_t x, int32_t y) { return x > y ? x : y; });
}

// The tile of workgroup `slot`: of 64 segments the tiles in falling order of their number, `forward`, or of how many follow, where the
// first ones' walks are the longest. A workgroup without one gets a segment of no tokens.
template <int SIZE> __device__ __forceinline__ Segment segment_of(const Packed &a, int32_t slot, int32_t unit, bool forward)
{
    const int32_t lane = (int32_t)threadIdx.x & 63, segments = a.sequences + 2;
    int32_t lo = 0, len = (segments + 63) / 64; // of 64 segments each: the last that begins at or in front of the slot
    while (len > 1) {
        const int32_t step = (len + 63) / 64, i = lo + lane * step;
        const uint64_t found = __ballot(lane * step < len && place_of<SIZE>(boundary(a, 64 * i), unit, 64 * i) <= slot) | 1u;
        const int32_t j = 63 - __builtin_clzll(found);
        lo += j * step;
        len = len - j * step < step ? len - j * step : step;
    }
    const int32_t mine = 64 * lo + lane, begin = boundary(a, mine), end = boundary(a, mine + 1);
    const int32_t count = mine < segments && end > begin ? end - begin : 0, tiles = (int32_t)(((int64_t)count * unit + SIZE - 1) / SIZE);
    const int32_t rank = slot - place_of<SIZE>(__builtin_amdgcn_readfirstlane(begin), unit, 64 * lo);
    // the largest number that more than `rank` tiles have or exceed
    int32_t number = 0;
    auto from = [&](int32_t n) { return sum_of_lanes(tiles > n ? tiles - n : 0); };
    const bool there = rank >= 0 && from(0) > rank;
    if (there) {
        int32_t above = largest_of_lanes(tiles); // none has more
        while (above - number > 1) {
            const int32_t n = number + (above - number) / 2;
            if (from(n) > rank)
                number = n;
            else
                above = n;
        }
    }
    const int32_t turn = rank - from(number + 1);
    const uint64_t have = __ballot(tiles > number);
    const uint64_t below = have & (((uint64_t)1 << lane) - 1u);
    const uint64_t found = __ballot(tiles > number && __popcll(below) == turn);
    const int32_t at = found ? __builtin_ctzll(found) : 0;
    Segment s;
    s.first = __builtin_amdgcn_readlane(begin, at);
    s.count = there ? __builtin_amdgcn_readlane(count, at) : 0;
    s.tile = !there ? 0 : forward ? number : __builtin_amdgcn_readlane(tiles, at) - 1 - number;
    s.index = 64 * lo + at;
    s.none = s.index == 0 || s.index == segments - 1;
    return s;
}

// Row r of a segment: where it is among a key head's rows, and in [tokens, heads, dim] in bytes.
__device__ __forceinline__ int64_t packed_row(const Packed &a, const Segment &s, int64_t row) { return (int64_t)s.first * a.group + row; }
__device__ __forceinline__ int64_t packed_at(const Packed &a, const Segment &s, int32_t kvh, uint32_t row)
{
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    return 2 * ((int64_t)s.first * heads_dim + (int64_t)kvh * a.group * a.dim + row_offset(row, (uint32_t)a.group, heads_dim, a.dim));
}

// Tiles of ROWS tokens, as TileLoads, where what lies behind the last one is cut off by the diagonal in any case: the last one once more
// takes its place. Pieces of channels that are not there are not loaded: their places in LDS are cleared once.  So every load has the
// tile's address in scalar registers and 32 bits of a lane's own; loads with an address each, and zeros to read, take eight registers more,
// which the kernel of 64 channels has not got.
template <int DP, int ROWS, int WAVES> struct LastTwiceLoads {
    static constexpr int kChunks = DP / 8, kLoads = ROWS * kChunks / 64, kMine = kLoads / WAVES;
    static_assert(kMine * WAVES == kLoads, "");
    uint32_t offset[kMine];
    uint32_t first, there; // there: bit q, whether the lane's piece of load q is

    __device__ __forceinline__ uint32_t row(int q, uint32_t lane) const { return ((first + (uint32_t)(q * WAVES)) * 64u + lane) / kChunks; }
    __device__ __forceinline__ uint32_t chunk(int q, uint32_t lane) const
    {
        return (((first + (uint32_t)(q * WAVES)) * 64u + lane) % kChunks) ^ swizzle<DP>(row(q, lane));
    }
    __device__ __forceinline__ LastTwiceLoads(int wave, int lane, int64_t token_stride, int32_t dim) : first((uint32_t)wave), there(0)
    {
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            offset[q] = row(q, (uint32_t)lane) * (uint32_t)token_stride + chunk(q, (uint32_t)lane) * 16u;
            there |= chunk(q, (uint32_t)lane) * 8u < (uint32_t)dim ? 1u << q : 0u;
        }
    }
    // the pieces that are not there, in a tile's place
    __device__ __forceinline__ void clear(int lane, uint32_t lds_at) const
    {
#pragma unroll
        for (int q = 0; q < kMine; ++q)
            if (!(there >> q & 1u))
                lds_write16(lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP> + 16u * (uint32_t)lane, u32x4{});
    }
    // load q of a tile that is there as a whole, from `base`, in scalar registers
    __device__ __forceinline__ void one(int q, uint64_t base, uint32_t lds_at) const
    {
        load_to_lds(base, offset[q], lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
    }
    // base: the tile's first token; rows: tokens that are there, from 1 on
    __device__ __forceinline__ void issue(uint64_t base, int64_t token_stride, int32_t dim, int32_t rows, uint32_t lds_at) const
    {
        const uint64_t from = uniform_u64(base);
        if (dim == DP && rows >= ROWS) { // (apart, without a branch between them)
#pragma unroll
            for (int q = 0; q < kMine; ++q)
                one(q, from, lds_at);
            return;
        }
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t l = lane_here();
            const uint32_t r = row(q, l), o = (r < (uint32_t)rows ? r : (uint32_t)rows - 1) * (uint32_t)token_stride + chunk(q, l) * 16u;
            if (there >> q & 1u)
                load_to_lds(from, o, lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
        }
    }
};

// The same of ROWS rows of the list, whose places are their queries' and their heads': rows behind the last one of a segment are its last
// one once more (their probabilities are set to zero).  Where a tile holds whole queries the places in it are the same in every tile;
// elsewhere they are computed anew for each.
template <int DP, int ROWS, int WAVES> struct RowsTwiceLoads {
    static constexpr int kChunks = DP / 8, kLoads = ROWS * kChunks / 64, kMine = kLoads / WAVES;
    static_assert(kMine * WAVES == kLoads, "");
    uint32_t offset[kMine];
    uint32_t first, there;

    __device__ __forceinline__ uint32_t row(int q, uint32_t lane) const { return ((first + (uint32_t)(q * WAVES)) * 64u + lane) / kChunks; }
    __device__ __forceinline__ uint32_t chunk(int q, uint32_t lane) const
    {
        return (((first + (uint32_t)(q * WAVES)) * 64u + lane) % kChunks) ^ swizzle<DP>(row(q, lane));
    }
    __device__ __forceinline__ RowsTwiceLoads(int wave, int lane, const Operand &o, const Packed &a) : first((uint32_t)wave), there(0)
    {
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            offset[q] = (uint32_t)row_offset(row(q, (uint32_t)lane), (uint32_t)a.group, o.token, o.head) + chunk(q, (uint32_t)lane) * 16u;
            there |= chunk(q, (uint32_t)lane) * 8u < (uint32_t)a.dim ? 1u << q : 0u;
        }
    }
    __device__ __forceinline__ void clear(int lane, uint32_t lds_at) const
    {
#pragma unroll
        for (int q = 0; q < kMine; ++q)
            if (!(there >> q & 1u))
                lds_write16(lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP> + 16u * (uint32_t)lane, u32x4{});
    }
    // base: the segment's first row; rows: of the segment
    __device__ __forceinline__ void issue(const Operand &o, uint64_t base, int32_t t, int32_t rows, const Packed &a, uint32_t lds_at) const
    {
        const uint32_t group = (uint32_t)a.group, row0 = (uint32_t)t * ROWS, query0 = row0 / group;
        const uint64_t from = uniform_u64(base + (uint64_t)query0 * (uint64_t)o.token);
        if (a.dim == DP && ROWS % group == 0 && row0 + ROWS <= (uint32_t)rows) {
#pragma unroll
            for (int q = 0; q < kMine; ++q)
                load_to_lds(from, offset[q], lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
            return;
        }
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t l = lane_here();
            const uint32_t r = row0 + row(q, l), mine = r < (uint32_t)rows ? r : (uint32_t)rows - 1, query = mine / group;
            const uint32_t place = (query - query0) * (uint32_t)o.token + (mine - query * group) * (uint32_t)o.head + chunk(q, l) * 16u;
            if (there >> q & 1u)
                load_to_lds(from, place, lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
        }
    }
};

// host
grkan_status_t fill(const grkan_causal_attention_t *a, grkan_dtype_t io, Packed *to); // checks and arguments (grkan_causal.hip)
bool few_rows(const Packed &a); // whether two wavefronts share the keys of 32 rows (grkan_causal.hip)
template <int SIZE> inline int64_t slots_of(const Packed &a, int64_t unit) { return (int64_t)a.tokens * unit / SIZE + a.sequences + 2; }

} // namespace attention
} // namespace grkan
#endif // GRKAN_PACKED_H_
