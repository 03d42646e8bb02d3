// What the backward kernels of attention share: tiles of rows, the largest of a wavefront's numbers, and float16's scales.
#ifndef GRKAN_ATTENTION_BACK_H_
#define GRKAN_ATTENTION_BACK_H_

#include "grkan_attention.h"

namespace grkan {
namespace attention {

constexpr int kRowTile = 64;

// Tiles of ROWS rows of the list: as TileLoads, but a row's place is its query's and its head's.  Where a tile holds whole queries, the
// places in it are the same in every tile; elsewhere they are computed anew for each.
template <int DP, int ROWS, int WAVES> struct RowLoads {
    static constexpr int kChunks = DP / 8, kLoads = ROWS * kChunks / 64, kMine = kLoads / WAVES;
    static_assert(kLoads % WAVES == 0, "");
    uint32_t offset[kMine], row[kMine], chunk[kMine]; // chunk: its bytes, or ~0: no such channels
    int first;
    bool even;
    uint64_t base, advance; // (even) of a tile

    __device__ __forceinline__ RowLoads(int wave, int lane, const Operand &o, uint64_t base_, bool even_, const Args &a)
        : first(wave), even(even_), base(base_)
    {
        const uint32_t group = (uint32_t)a.group;
        advance = even ? (uint64_t)(ROWS / group) * (uint64_t)o.token : 0;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t e = (uint32_t)(first + q * WAVES) * 64u + (uint32_t)lane;
            row[q] = e / kChunks;
            const uint32_t c = (e % kChunks) ^ swizzle<DP>(row[q]);
            chunk[q] = c * 8u < (uint32_t)a.dim ? c * 16u : ~0u;
            offset[q] = (uint32_t)row_offset(row[q], group, o.token, o.head) + c * 16u;
        }
    }
    __device__ __forceinline__ void issue(const Operand &o, int32_t t, int64_t rows, const Args &a, uint32_t lds_at) const
    {
        const uint32_t row0 = (uint32_t)t * ROWS;
        const uint64_t tile = base + (uint64_t)(uint32_t)t * advance;
        const bool whole = even && a.dim == DP && (int64_t)row0 + ROWS <= rows;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t to = lds_at + (uint32_t)(first + q * WAVES) * kBlock<DP>;
            if (whole) {
                load_to_lds(uniform_u64(tile), offset[q], to);
            } else {
                uint32_t r = row[q];
                keep_in_loop(r);
                const bool there = (int64_t)row0 + r < rows && chunk[q] != ~0u;
                const uint64_t at = even ? tile + offset[q] : base + (uint64_t)row_offset(row0 + r, (uint32_t)a.group, o.token, o.head) + chunk[q];
                load_to_lds_at(there ? at : reinterpret_cast<uint64_t>(kZeros), to);
            }
        }
    }
};

// 4 bytes a lane to LDS bytes lds_at + 4 lane ..
__device__ __forceinline__ void load_words_to_lds(uint64_t base, uint32_t lane_off, uint32_t lds_at)
{
    asm volatile("s_nop 4\n\tglobal_load_lds_dword %1, %2" : : "{m0}"(lds_at), "v"(lane_off), "s"(base) : "memory");
}

// The largest of a wavefront's numbers (none negative), as bits, in all lanes.  (In registers: the keys' kernel has three of these in front of a walk
// that may be short.  4 x 64 queries, 16,000 keys, eight heads of 128 that read two, float16: 150 us with shuffles through LDS and more loads, 145 so.)
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t bits)
{
    auto with = [&](uint32_t o) { bits = o > bits ? o : bits; };
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2 of four
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0x4e, 0xf, 0xf, true));  // 2 3 0 1
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0x141, 0xf, 0xf, true)); // eight mirrored
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)bits, 0x140, 0xf, 0xf, true)); // sixteen mirrored
    const auto rows = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    bits = rows[0] > rows[1] ? rows[0] : rows[1];
    const auto halves = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    return halves[0] > halves[1] ? halves[0] : halves[1];
}
__device__ __forceinline__ uint32_t greater(uint32_t bits, float v)
{
    const uint32_t o = __builtin_bit_cast(uint32_t, v);
    return o > bits ? o : bits;
}

// float16's rows come first: their scales are needed in front of the products.
template <typename IO> constexpr bool kRowsFirst = !__is_same(IO, __bf16);

// 2^e for the largest |dO| (its bits; 1 where that is zero or not finite)
__device__ __forceinline__ float scale_of(uint32_t bits)
{
    // (dO is float16: its exponent is -24 .. 15)
    const int e = (int)(bits >> 23) - 127 + 2;
    return bits == 0 || e > 17 ? 1.0f : __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
}

// 2^e lowered, where what it multiplies may pass 32,768 otherwise: sqrt(dim) / 2 for each unit of a value's length (squared: length2), and `up` sums
// (where they are not finite: not)
__device__ __forceinline__ float lowered(float up, float length2, float sums, int32_t dim)
{
    const float most = 0.5f * sqrtf(length2 * (float)dim) + up * sums;
    const int e = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - 15; // 2^(e + 15) .. 2^(e + 16)
    return e < 0 || e > 100 ? up : up * __builtin_bit_cast(float, (uint32_t)(127 - (e + 1)) << 23);
}

// ROWS: of a stage of the keys' kernel.  V_LDS: that kernel reads V from LDS at every use; its registers hold K and the sums alone.
template <typename IO_, int DP_, int ROWS_, bool V_LDS_, int PER_> struct BackShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, ROWS = ROWS_, PER = PER_, kWaves = 4;
    static constexpr bool V_LDS = V_LDS_;
    static constexpr int kOwn = 32 * kWaves; // keys or rows of a workgroup
    static_assert(kOwn == kGroup, "");
    // keys' kernel: Q, dO, lse, delta of ROWS rows; queries' kernel: K, V of 64 keys
    static constexpr uint32_t kRowsTile = kTileBytes<DP, ROWS>, kKeyStage = 2 * kRowsTile + 2 * ROWS * 4u;
    static constexpr uint32_t kKeysTile = kTileBytes<DP, 64>, kRowStage = 2 * kKeysTile, kCover = 2 * kRowStage; // and behind two of those what covers keys
    static constexpr size_t kKeyLds = 2 * (size_t)kKeyStage + (V_LDS ? 2 * (size_t)kKeysTile : 0), kRowLds = kCover + 2 * 64 * 4;
};

} // namespace attention
} // namespace grkan
#endif // GRKAN_ATTENTION_BACK_H_
