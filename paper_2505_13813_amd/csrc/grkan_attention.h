// What the cross attention's kernels share: arguments, tiles of rows in LDS, and operands of the matrix instructions from them.
//
// The queries of the heads that read one key head are one list of rows: row r is query r / group of head r mod group, so that every
// product has as many rows as the heads allow, with one query too.
//
// All products run in 32 x 32 x 16 matrix instructions, arranged so that the probabilities never leave the registers: the scores
// are formed transposed, S^T = K Q^T, and a lane then holds sixteen keys of one row (keys 8 (i / 4) + 4 (lane / 32) + i mod 4);
// the order of the keys in a contraction is free as long as both operands agree, and in this one the lane's probabilities are
// the second operand of V^T P^T as they lie.  V^T comes from V's rows in LDS by transposing reads, numbered the same way.
#ifndef GRKAN_ATTENTION_H_
#define GRKAN_ATTENTION_H_

#include "../../include/grkan_transformer.h"
#include "grkan_tile.h"

namespace grkan {
namespace attention {

using namespace tile;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// [batch, token, head, channel]; strides in bytes
struct Operand {
    uint64_t at;
    int64_t batch, token, head;
};

struct Args {
    Operand q, k, v, dout;
    const void *lengths;
    const uint8_t *mask;
    int64_t mask_batch, mask_key;
    int64_t keys, rows; // rows: queries x group
    int32_t batch, kv_heads, group, dim;
    int32_t lengths_64;
    float c; // scale x log2(e)
    float scale;
    char *out;              // dq in the backward pass
    uint64_t forward_out;   // the backward pass' second input
    char *dk, *dv;
    float *lse;             // [batch, kv_heads, rows]
    float *partial;         // [splits][batch, kv_heads][rows][dim], then the splits' lse [splits][batch, kv_heads][rows]
    // backward: of each row, padded to whole tiles of 64, its lse and sum over channels of dout out; float16: of each 64 rows the largest |dout| and
    // the largest |sum|, of each 32 keys the largest sum over channels of v^2
    float *row_lse, *row_delta, *row_most, *value_most;
    int32_t padded;         // rows with the padding
    int32_t even_q, even_dout; // places of a tile's rows in q and dout in 32 bits
    int32_t splits, tiles_per_split; // (splits: the workers, where the groups of keys are dealt out; the most parts, in the keys' gradients)
    int32_t row_tiles, key_tiles; // workgroups of a key head over rows, over keys
    int32_t at_once;       // workgroups of the keys' gradients that the device holds
    int32_t work, run; // work items, and how many of them in a row one XCD gets
};

// Instruction kinds of __builtin_amdgcn_sched_group_barrier.
constexpr int kProducts = 0x8, kLdsReads = 0x100;

template <typename IO> struct Matrix;
template <> struct Matrix<__bf16> {
    static __device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 multiply16(const u32x4 &a, const u32x4 &b, const f32x4 &c) // 16 x 16 x 32
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t two(float a, float b) { return pack(a, b); }
    static __device__ __forceinline__ float first(uint32_t w) { return low(w); }
    static __device__ __forceinline__ float second(uint32_t w) { return high(w); }
};
template <> struct Matrix<_Float16> {
    static __device__ __forceinline__ f32x16 multiply(const u32x4 &a, const u32x4 &b, const f32x16 &c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 multiply16(const u32x4 &a, const u32x4 &b, const f32x4 &c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        f32x2 v;
        v[0] = a;
        v[1] = b;
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
    static __device__ __forceinline__ float first(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
    static __device__ __forceinline__ float second(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
};

// Row r of a key head's list: query r / group of its head r mod group.
__device__ __forceinline__ int64_t row_offset(uint32_t row, uint32_t group, int64_t token, int64_t head)
{
    if (group == 1)
        return (int64_t)row * token;
    const uint32_t query = row / group;
    return (int64_t)query * token + (int64_t)(row - query * group) * head;
}

// Where loads of rows and channels that are not there read: zeros, so that nothing that lies in memory behind them (NaN times a
// probability of zero is NaN) gets into a product.
static __device__ const uint4 kZeros[16] __attribute__((aligned(256))) = {};

// A tile's rows in LDS.  16-byte pieces are permuted within a row, piece p of row r at slot p ^ swizzle(r), and, with rows of 128 or 256 bytes, every
// KB is followed by 16 bytes of nothing, so that the reads of both kinds hit all 64 banks at once: the same piece of sixteen rows one behind
// the other, and four adjacent pieces of four rows.  (Measured: a row operand's read 4.5 cycles of a compute unit, a column operand's 2.7; with rows
// permuted for eight rows and for two pieces, as the counters of conflicts have it 8.4 and 4.1.)
template <int DP> __device__ __forceinline__ constexpr uint32_t swizzle(uint32_t row)
{
    return DP == 128 ? 4u * (row & 3u) : DP == 64 ? 2u * (row & 2u) + ((row & 4u) >> 1) : (row >> 2) & 3u;
}
template <int DP> constexpr uint32_t kBlock = DP == 64 || DP == 128 ? 1040u : 1024u; // what a wavefront loads at once
template <int DP> __device__ __forceinline__ constexpr uint32_t row_at(uint32_t row)
{
    return row * DP * 2u + (DP == 64 || DP == 128 ? row * DP * 2u / 1024u * 16u : 0u);
}
template <int DP, int ROWS> constexpr uint32_t kTileBytes = ROWS *DP * 2u / 1024u * kBlock<DP>;

// 16 bytes a lane from its own address to LDS bytes lds_at + 16 lane .. (as load_to_lds, with addresses instead of offsets)
__device__ __forceinline__ void load_to_lds_at(uint64_t address, uint32_t lds_at)
{
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds_at), "v"(address) : "memory");
}

// Loads into registers have arrived, behind this: the compiler, which does not know of the loads to LDS, would else wait for all of
// those too at every use of the registers in the loop behind.
template <int N> __device__ __forceinline__ void arrived(u32x4 (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+v"(r[i]));
}
__device__ __forceinline__ void arrived(float &r) { asm volatile("" : "+v"(r)); }

// The lane's number, computed where it is asked for: for loops that have no register to keep it in.
__device__ __forceinline__ uint32_t lane_here()
{
    uint32_t lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    return lane;
}

__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// Tiles of ROWS tokens (keys) by WAVES wavefronts, a KB at a time.  Where one wavefront loads a tile by itself, in a loop: that kernel is over in
// microseconds, and waits for its own code, which comes to every compute unit with the launch (its first loads are out after 2.2 us of a wavefront's
// life; with eight loads written out 4.7).  Where four do, written out: 220 us in the place of 242 for 2 x 4096 x 4001 of 16 heads of 128.
template <int DP, int ROWS, int WAVES> struct TileLoads {
    static constexpr int kChunks = DP / 8, kLoads = ROWS * kChunks / 64, kMine = kLoads / WAVES;
    // loads kEach WAVES apart differ by whole tokens alone: the pieces of a row are permuted alike in both
    static constexpr int kEach = WAVES > 1 ? kMine : DP == 96 ? 3 : 1, kTurns = kMine / kEach;
    static constexpr uint32_t kTokens = (uint32_t)(kEach * WAVES * 64 / kChunks); // between them
    static_assert(kMine * WAVES == kLoads && kTurns * kEach == kMine && kEach * WAVES * 64 % kChunks == 0, "");

    uint32_t offset[kEach], row[kEach]; // of the first turn: bytes from the tile's first row; the row, or 64: no such channels
    uint32_t first;

    __device__ __forceinline__ TileLoads(int wave, int lane, int64_t token_stride, int32_t dim) : first((uint32_t)wave)
    {
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const uint32_t e = (first + (uint32_t)(q * WAVES)) * 64u + (uint32_t)lane;
            const uint32_t r = e / kChunks, chunk = (e % kChunks) ^ swizzle<DP>(r);
            offset[q] = r * (uint32_t)token_stride + chunk * 16u;
            row[q] = chunk * 8u < (uint32_t)dim ? r : 64u;
        }
    }

    // base: the tile's first row (the same in all lanes); word: which rows are valid; whole: all of them, and all channels
    __device__ __forceinline__ void issue(uint64_t base, int64_t token_stride, uint64_t word, bool whole, uint32_t lds_at) const
    {
        const uint64_t step = (uint64_t)token_stride * kTokens;
        uint32_t to = lds_at + first * kBlock<DP>;
#pragma unroll 1
        for (int turn = 0; turn < kTurns; ++turn) {
#pragma unroll
            for (int q = 0; q < kEach; ++q) {
                if (whole) {
                    load_to_lds(uniform_u64(base), offset[q], to);
                } else {
                    const bool there = row[q] < 64u && ((word >> (row[q] & 63u)) & 1u);
                    load_to_lds_at(there ? base + offset[q] : reinterpret_cast<uint64_t>(kZeros), to);
                }
                to += WAVES * kBlock<DP>;
            }
            if constexpr (kTurns > 1) {
                base += step;
                word >>= kTokens;
            }
        }
    }
};

// Addresses of a lane, moved to a tile.  (The compiler is kept from adding the tile's place to each read's constant part instead, which
// takes an instruction for every read.)
template <int N> struct Addresses {
    uint32_t at[N];
    __device__ __forceinline__ Addresses moved(uint32_t tile) const
    {
        Addresses r;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            r.at[i] = at[i] + tile;
            asm volatile("" : "+v"(r.at[i]));
        }
        return r;
    }
    // the same in place: for loops that have no registers for both
    __device__ __forceinline__ void move(uint32_t by)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            at[i] += by;
            asm volatile("" : "+v"(at[i]));
        }
    }
};

// First operand from a tile's rows: lane l has row 32 block + l mod 32, channels 16 step + 8 (l / 32) ..
template <int DP> struct RowOperand : Addresses<DP / 16> {
    __device__ __forceinline__ explicit RowOperand(int lane)
    {
        const uint32_t row = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
            this->at[s] = row_at<DP>(row) + (((uint32_t)(2 * s) + h) ^ swizzle<DP>(row)) * 16u;
    }
    // `further`: of a second tile, that many bytes behind
    static __device__ __forceinline__ u32x4 read(const Addresses<DP / 16> &from, int block, int step, uint32_t further = 0)
    {
        return lds_read16(from.at[step] + (row_at<DP>(32u * block) + further));
    }
};

// First operand from a tile's columns: lane l has channel 32 part + l mod 32 and, of the sixteen rows 32 block + 16 t .., those that the
// lane's sums hold: 4 (l / 32) .. + 3 and 8 + 4 (l / 32) .. + 3
template <int DP> struct ColumnOperand : Addresses<DP / 32> {
    __device__ __forceinline__ explicit ColumnOperand(int lane)
    {
        const uint32_t i = (uint32_t)lane & 15u, part16 = ((uint32_t)lane >> 4) & 1u, h = (uint32_t)lane >> 5;
        const uint32_t row = 4u * h + (i >> 2);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
            this->at[d] = row_at<DP>(row) + ((4u * d + 2u * part16 + ((i & 3u) >> 1)) ^ swizzle<DP>(row)) * 16u + (i & 1u) * 8u;
    }
    static __device__ __forceinline__ u32x4 read(const Addresses<DP / 32> &from, int block, int t, int part, uint32_t further = 0)
    {
        // (eight rows further the pieces are permuted alike, but for the short and the uneven rows)
        constexpr uint32_t flip = swizzle<DP>(8u) * 16u;
        const uint32_t first = from.at[part] + (row_at<DP>(32u * block + 16u * t) + further);
        const uint32_t second = (flip ? from.at[part] ^ flip : from.at[part]) + (row_at<DP>(32u * block + 16u * t + 8u) + further);
        const u32x2 a = __builtin_bit_cast(u32x2, lds_read_transposed(first)), b = __builtin_bit_cast(u32x2, lds_read_transposed(second));
        u32x4 r;
        r[0] = a[0];
        r[1] = a[1];
        r[2] = b[0];
        r[3] = b[1];
        return r;
    }
};

// The same of both halves of a wavefront (lanes l and l + 32 hold parts of one row).
__device__ __forceinline__ float halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// The same of the four lanes l mod 16, l mod 16 + 16, ..
__device__ __forceinline__ float quarters_max(float v)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    return halves_max(fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])));
}
__device__ __forceinline__ float quarters_sum(float v)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    return halves_sum(__builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]));
}

__device__ __forceinline__ int32_t keys_of(const Args &a, int32_t b)
{
    if (!a.lengths)
        return (int32_t)a.keys;
    const int64_t n = a.lengths_64 ? static_cast<const int64_t *>(a.lengths)[b] : (int64_t) static_cast<const int32_t *>(a.lengths)[b];
    return (int32_t)(n < 0 ? 0 : n < a.keys ? n : a.keys);
}

// Which keys of a batch entry are valid, 64 to a word, up to word `end`.  With a mask, lane i keeps word first + i, and the words are made 64 at a time, or as many
// as there are: sixteen loads out at once, and no branch between them.  (One token, 6,277 keys, twelve heads that read six of 64 channels, batch of 2:
// 22 us with eight at once and always 64 words, 12 so.)
struct ValidKeys {
    const uint8_t *mask;
    int64_t stride;
    int32_t count, end, first;
    uint64_t mine;

    __device__ __forceinline__ ValidKeys(const Args &a, int32_t b, int32_t count_, int32_t end_)
        : mask(a.mask ? a.mask + (int64_t)b * a.mask_batch : nullptr), stride(a.mask_key), count(count_), end(end_), first(-64), mine(0)
    {
    }
    // word w < end: keys 64 w .. (asked in rising order, by all lanes; the first of them below count)
    __device__ __forceinline__ uint64_t word(int32_t w)
    {
        const int32_t left = count - 64 * w;
        const uint64_t below = left >= 64 ? ~(uint64_t)0 : left > 0 ? ((uint64_t)1 << left) - 1u : 0u;
        if (!mask)
            return below;
        if (w - first >= 64) {
            const int lane = (int)threadIdx.x & 63;
            first = w;
            const int words = end - w < 64 ? end - w : 64;
#pragma unroll 1
            for (int i0 = 0; i0 < words; i0 += 16) {
                uint8_t m[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int64_t key = 64 * ((int64_t)w + i0 + i) + lane;
                    m[i] = mask[(key < count ? key : 0) * stride];
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) { // (keys from `count` on are cut off below)
                    const uint64_t found = __ballot(m[i] != 0);
                    mine = i0 + i == lane ? found : mine;
                }
            }
        }
        const int from = w - first;
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, from);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), from);
        return below & (((uint64_t)hi << 32) | lo);
    }
};

// What is added to the scores of a tile's keys, in LDS: 0, or minus infinity where a key is not valid.  The matrix instructions start from it, so that
// a mask takes no vector instruction for each score (a bit test, a comparison, a selection and a wait).
__device__ __forceinline__ void write_cover(uint32_t at, uint64_t word, int lane)
{
    *(__attribute__((address_space(3))) float *)(uintptr_t)(at + 4u * (uint32_t)lane) = (word >> lane) & 1u ? 0.0f : -__builtin_inff();
}
// of 32 keys, as the scores lie in the lanes
__device__ __forceinline__ f32x16 read_cover(uint32_t at, int block, uint32_t h)
{
    f32x16 r;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 c = __builtin_bit_cast(f32x4, lds_read16(at + (32u * block + 8u * g + 4u * h) * 4u));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[4 * g + j] = c[j];
    }
    return r;
}

// The keys of all key heads one behind the other, in groups of 128 that do not reach over a head's end: who deals them out evenly to its
// workers gives all the same to do, whatever the batch entries' lengths are.
// (Everything in 32 bits: the host lets no more than 2^30 groups come here.)
constexpr int kGroup = 128;
// How many walks over an entry's keys there are: its key heads.
__device__ __forceinline__ int32_t units_of(const Args &a) { return a.kv_heads; }

// GROUP: keys of a group.
template <class A, int GROUP = kGroup> struct DealOf {
    int32_t total, workers; // G, and W: as many as the host asked for, but none without a group
    int32_t quotient, rest; // of G by W
    // batch entry b, its keys, the groups of one of its key heads, and the group that its first one begins with
    int32_t b, count, groups, begin;
    int32_t mine, up_to; // of entry `lane`: its keys; the groups up to and with it, of one key head each

    __device__ __forceinline__ static int32_t groups_of(int32_t keys) { return (keys + GROUP - 1) / GROUP; }

    // keys of entry first + lane (0 behind the last), and the running sum of the groups
    __device__ __forceinline__ static void scan(const A &a, int32_t first, int32_t &keys, int32_t &sum)
    {
        const int32_t lane = (int32_t)threadIdx.x & 63, entry = first + lane;
        keys = entry < a.batch ? keys_of(a, entry) : 0;
        sum = groups_of(keys);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t o = __shfl_up(sum, d);
            sum += lane >= d ? o : 0;
        }
    }

    __device__ __forceinline__ explicit DealOf(const A &a)
    {
        if (!a.lengths) {
            total = groups_of((int32_t)a.keys) * units_of(a) * a.batch;
        } else {
            scan(a, 0, mine, up_to);
            total = __builtin_amdgcn_readlane(up_to, 63);
            for (int32_t first = 64; first < a.batch; first += 64) {
                int32_t keys, sum;
                scan(a, first, keys, sum);
                total += __builtin_amdgcn_readlane(sum, 63);
            }
            total *= units_of(a);
        }
        workers = total < a.splits ? total : a.splits;
        quotient = workers ? total / workers : 0;
        rest = total - quotient * workers;
    }
    // worker w's first group, w G / W
    __device__ __forceinline__ int32_t first_of(int32_t w) const { return w * quotient + w * rest / workers; }
    // the worker that has group x
    __device__ __forceinline__ int32_t worker_of(int32_t x) const
    {
        int32_t w = (int32_t)((float)x * ((float)workers / (float)total));
        w = w < workers ? w : workers - 1;
        while (first_of(w) > x)
            --w;
        while (first_of(w + 1) <= x)
            ++w;
        return w;
    }
    // Sets b, count, groups and begin: to the entry that holds group x, or to `entry`.
    __device__ __forceinline__ void find(const A &a, int32_t x, int32_t entry = -1)
    {
        if (!a.lengths) {
            count = (int32_t)a.keys;
            groups = groups_of(count);
            b = entry >= 0 ? entry : x / (groups * units_of(a));
            begin = b * groups * units_of(a);
            return;
        }
        int32_t before = 0; // groups of a key head each, of the entries in front
        for (int32_t first = 0;; first += 64) {
            int32_t keys = mine, sum = up_to;
            if (first)
                scan(a, first, keys, sum);
            const int32_t lane = (int32_t)threadIdx.x & 63;
            const uint64_t found = __ballot(entry >= 0 ? first + lane == entry : (before + sum) * units_of(a) > x);
            if (found || first + 64 >= a.batch) {
                const int at = found ? __builtin_ctzll(found) : 63;
                b = first + at;
                count = __builtin_amdgcn_readlane(keys, at);
                groups = groups_of(count);
                begin = (before + __builtin_amdgcn_readlane(sum, at) - groups) * units_of(a);
                return;
            }
            before += __builtin_amdgcn_readlane(sum, 63);
        }
    }
};
typedef DealOf<Args> Deal;

// Workgroups go round-robin over the 8 XCDs.  Runs of work items go to one XCD, whose L2 fetches their keys and values once; runs
// are short enough (host: spread) that every XCD has several of them, of long and of short batch entries.
__device__ __forceinline__ int32_t work_item(const Args &a)
{
    const int32_t xcd = (int32_t)blockIdx.x & 7, i = (int32_t)blockIdx.x >> 3;
    const int32_t turn = i / a.run;
    return (turn * 8 + xcd) * a.run + (i - turn * a.run);
}

// host
grkan_status_t fill(const grkan_attention_t *a, grkan_dtype_t io, Args *to); // checks and arguments (grkan_attention.hip)
bool allow_lds(const void *kernel, size_t bytes);
bool in_offsets(int64_t token_stride, int64_t head_stride, int64_t heads);    // of a tile, in elements of 2 bytes
constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1;  // of 256 threads: a launch has less than 2^32
int64_t spread(Args &a, int64_t work, int64_t per_head); // sets work (kMostBlocks at most) and run; the grid, which may be more
int64_t splits_of(int64_t base, int64_t tiles, int64_t rows, int64_t dim, double together, double tile); // of a walk over the keys

} // namespace attention
} // namespace grkan
#endif // GRKAN_ATTENTION_H_
