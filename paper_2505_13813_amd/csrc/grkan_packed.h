// Sequences packed one behind the other, each attending to its own earlier tokens: what the forward and the backward kernels share.
//
// The buffer's tokens fall into segments: those in front of the first sequence, the sequences, those behind the last.  A workgroup has a tile of one segment,
// `size` rows that begin with the segment's.  Tile t of a segment that begins with row r (of all rows of a key head) and is number i has slot
// floor(r / size) + i + t: the segments' slots do not overlap (floor(x + y) >= floor(x) + floor(y)), there are at most floor(rows / size) + segments of them,
// and which segment a slot belongs to is found by a search in the offsets, without sums over the lengths, a launch in front or the host's knowing them.
// A slot without rows has nothing to do.
#ifndef GRKAN_PACKED_H_
#define GRKAN_PACKED_H_

#include "grkan_attention.h"

namespace grkan {
namespace attention {

struct Packed : Args { // rows: of all tokens; batch and the operands' batch strides: not used
    const void *offsets;
    int32_t offsets_64, sequences;
    int32_t tokens, each; // each: of a sequence, where there are no offsets
    int32_t slots;        // workgroups of a key head
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

// unit: rows of a token.  Offsets that fall give slots whose tokens are unspecified, but within the buffer.
template <int SIZE> __device__ __forceinline__ int32_t slot_of(int32_t token, int32_t unit, int32_t i)
{
    return (int32_t)((uint32_t)token * (uint32_t)unit / (uint32_t)SIZE) + i;
}
template <int SIZE> __device__ __forceinline__ Segment segment_of(const Packed &a, int32_t slot, int32_t unit)
{
    const int32_t lane = (int32_t)threadIdx.x & 63;
    int32_t lo = 0, len = a.sequences + 2, begin = 0, end = 0;
    for (;;) {
        const int32_t step = (len + 63) / 64, i = lo + lane * step;
        const int32_t at = boundary(a, i < lo + len ? i : lo + len);
        const uint64_t found = __ballot(lane * step < len && slot_of<SIZE>(at, unit, i) <= slot) | 1u;
        const int32_t j = 63 - __builtin_clzll(found);
        lo += j * step;
        len = len - j * step < step ? len - j * step : step;
        if (len > 1)
            continue;
        begin = __builtin_amdgcn_readlane(at, j);
        end = j < 63 ? __builtin_amdgcn_readlane(at, j + 1) : __builtin_amdgcn_readfirstlane(boundary(a, lo + 1));
        break;
    }
    Segment s;
    s.first = begin;
    s.count = end > begin ? end - begin : 0;
    s.tile = slot - slot_of<SIZE>(begin, unit, lo);
    s.index = lo;
    s.none = lo == 0 || lo == a.sequences + 1;
    return s;
}

// Row r of a segment: where it is among a key head's rows, and in [tokens, heads, dim] in bytes.
__device__ __forceinline__ int64_t packed_row(const Packed &a, const Segment &s, int64_t row) { return (int64_t)s.first * a.group + row; }
__device__ __forceinline__ int64_t packed_at(const Packed &a, const Segment &s, int32_t kvh, uint32_t row)
{
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    return 2 * ((int64_t)s.first * heads_dim + (int64_t)kvh * a.group * a.dim + row_offset(row, (uint32_t)a.group, heads_dim, a.dim));
}

// Tiles of ROWS tokens, as TileLoads, where what lies behind the last one is cut off by the diagonal in any case: the last one once more takes its place.
// Pieces of channels that are not there are not loaded: their places in LDS are cleared once.  So every load has the tile's address in scalar registers and 32 bits
// of a lane's own; loads with an address each, and zeros to read, take eight registers more, which the kernel of 64 channels has not got.
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
    // base: the tile's first token; rows: tokens that are there, from 1 on
    __device__ __forceinline__ void issue(uint64_t base, int64_t token_stride, int32_t dim, int32_t rows, uint32_t lds_at) const
    {
        const uint64_t from = uniform_u64(base);
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            uint32_t o = offset[q];
            if (rows < ROWS) {
                const uint32_t l = lane_here();
                const uint32_t r = row(q, l);
                o = (r < (uint32_t)rows ? r : (uint32_t)rows - 1) * (uint32_t)token_stride + chunk(q, l) * 16u;
            }
            if (dim == DP || (there >> q & 1u))
                load_to_lds(from, o, lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
        }
    }
};

// The same of ROWS rows of the list, whose places are their queries' and their heads': rows behind the last one of a segment are its last one once more (their
// probabilities are set to zero).  Where a tile holds whole queries the places in it are the same in every tile; elsewhere they are computed anew for each.
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
        const bool whole = ROWS % group == 0 && row0 + ROWS <= (uint32_t)rows;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            uint32_t place = offset[q];
            if (!whole) {
                const uint32_t l = lane_here();
                const uint32_t r = row0 + row(q, l), mine = r < (uint32_t)rows ? r : (uint32_t)rows - 1, query = mine / group;
                place = (query - query0) * (uint32_t)o.token + (mine - query * group) * (uint32_t)o.head + chunk(q, l) * 16u;
            }
            if (a.dim == DP || (there >> q & 1u))
                load_to_lds(from, place, lds_at + (first + (uint32_t)(q * WAVES)) * kBlock<DP>);
        }
    }
};

// host
grkan_status_t fill(const grkan_causal_attention_t *a, grkan_dtype_t io, Packed *to); // checks and arguments (grkan_causal.hip)
template <int SIZE> inline int64_t slots_of(const Packed &a, int64_t unit) { return (int64_t)a.tokens * unit / SIZE + a.sequences + 2; }

} // namespace attention
} // namespace grkan
#endif // GRKAN_PACKED_H_
