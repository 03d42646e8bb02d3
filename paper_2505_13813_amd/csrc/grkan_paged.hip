// A cache of keys and values in pages, on gfx950 (MI355X): new tokens' keys and values into it, and attention of the newest tokens over it.
//
// Position p of sequence s lies in row p mod page_size of page table[s][p / page_size].  Of the `queries` newest tokens of a sequence of
// `length`, token i sees the positions up to length - queries + i: out_i = sum_p softmax_p(scale q_i k_p) v_p.
//
// The keys and values are read once, and that bounds it, as there are few rows for each: 32 sequences of 1 to 8,191 positions, 32 heads of
// 128 on 8, 592 MB, in 111 us = 5.4 TB/s, where reading alone gets 6.0.  A wavefront has tiles of 32 keys and their values by itself,
// without a barrier.  While it computes it loads little, and so the others must: eight wavefronts on a compute unit with 128 channels, a
// buffer each, do better than four with two (142 us; with everything in the cache, where only the way through a tile counts, 126, and 56
// so: the products have sixteen rows in place of 32, two wavefronts fill one another's waits).  The wavefronts side by side have the heads
// that lie side by side in memory (116 us with whole heads one behind the other).  Short walks are joined in their workgroup; long ones are
// dealt out evenly to all wavefronts, whatever the lengths are, and a second launch joins the parts. Where the pages are whole tiles a tile
// has one address; elsewhere every lane has its key's (pages of 16: 115 us).  The table's entries come to LDS in front of the walk, so that
// no load waits for another one within it.
#include <hip/hip_runtime.h>

#include <cmath>

#include "grkan_attention_rows.h"
#include "grkan_packed.h"

namespace grkan {
namespace attention {

struct Paged : Args { // keys: that a row of the table has place for; rows: queries x group; k, v: their `batch` is a page's stride
    const int32_t *table;
    int64_t table_stride;
    int64_t pages;
    int32_t page, entries; // tokens of a page; of a row of the table
    int32_t queries;
    int32_t tile_rows; // of a walk: 16 or 32
    int32_t unit_rows; // of a part: as many, or all where they are fewer
    int32_t bundle;     // walks that are dealt out together: 8, 4, 2 or 1
    int32_t join_lanes; // in the second launch: lanes of a row's piece
};

// Walks over a sequence's keys: each key head and tile of rows.  Where they are dealt out, `bundle` of them go together, a wavefront each.
__device__ __forceinline__ int32_t walks_of(const Paged &a) { return a.kv_heads * a.row_tiles; }
__device__ __forceinline__ int32_t units_of(const Paged &a) { return walks_of(a) / a.bundle; }

// Places for parts: worker w's of unit u is in u + w (no two are in the same: from one part to the next, one of the two rises).
__device__ __forceinline__ int64_t slots_of(const Paged &a) { return ((int64_t)a.batch * units_of(a) + a.splits) * a.bundle; }

constexpr int kTileKeys = 32;
constexpr int kEntries = 256; // of the table in LDS at once, for each wavefront
constexpr int kWaves = 8;     // of a workgroup

// BLOCKS: of sixteen rows.
template <typename IO_, int DP_, int BLOCKS_> struct PagedShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, BLOCKS = BLOCKS_, kRows = 16 * BLOCKS;
    static constexpr uint32_t kTile = kTileBytes<DP, kTileKeys>, kTable = 2 * kTile * kWaves;
    static constexpr size_t kLds = kTable + kWaves * kEntries * 4;
    static constexpr int kPitch = DP + 4; // of a row's channels, where the wavefronts join theirs
    static_assert((size_t)kWaves * kRows * (kPitch + 2) * sizeof(float) <= kLds, "");
    static constexpr int kPerUnit = BLOCKS == 1 && 2 * kLds <= 160 * 1024 ? 2 : 1; // workgroups of a compute unit
};

// A row's way over the pages: which keys of a tile there are, and its loads.  table: of positions from `first` x page on, in LDS, -1 where
// there is no page.
template <class SH> struct Pages {
    static constexpr int KT = kTileKeys, DP = SH::DP;
    using Loads = TileLoads<DP, KT, 1>;
    const Paged &a;
    const int32_t *table;
    const Loads &k_loads, &v_loads;
    uint64_t k_head, v_head;
    int lane;
    int32_t first, end; // the table's first entry; keys
    int32_t page, place; // where whole tiles are in a page: of the tile; else of key t KT + lane mod 32

    __device__ __forceinline__ bool even() const { return a.page % KT == 0; }

    __device__ __forceinline__ uint64_t word(int32_t t)
    {
        const int32_t left = end - t * KT;
        const uint64_t below = left >= KT ? 0xffffffffu : ((uint64_t)1 << left) - 1u;
        if (even()) {
            const int32_t entry = t * KT / a.page;
            page = __builtin_amdgcn_readfirstlane(table[entry - first]);
            place = t * KT - entry * a.page;
            return page >= 0 ? below : 0;
        }
        const int32_t key = t * KT + (lane & 31), entry = key / a.page;
        place = key - entry * a.page;
        page = key < end ? table[entry - first] : -1;
        return below & __ballot(page >= 0);
    }
    // keys or values (o, loads, head) of the tile that word() was asked for last
    __device__ __forceinline__ void load(const Operand &o, const Loads &loads, uint64_t head, uint64_t word, uint32_t to) const
    {
        // (every load written out: 1,000 positions, pages of 64, twelve heads of 64 channels 8.6 us in the place of 9.9 with a loop)
        if (even()) {
            uint64_t base = head + (page < 0 ? 0 : (uint64_t)page) * (uint64_t)o.batch + (uint64_t)place * (uint64_t)o.token;
            if (word != 0xffffffffu || a.dim != DP) {
                loads.issue(base, o.token, word, false, to);
                return;
            }
            base = uniform_u64(base);
#pragma unroll
            for (int n = 0; n < Loads::kMine; ++n)
                load_to_lds(base + (uint64_t)(n / Loads::kEach) * Loads::kTokens * (uint64_t)o.token, loads.offset[n % Loads::kEach], to + (uint32_t)n * kBlock<DP>);
            return;
        }
        // (all exchanges in front: they wait for one another otherwise.  The same on pages of 16 10.0 us in the place of 11.9, and 700 positions, 32
        // heads of 128 on eight, four sequences, 12.1 in the place of 14.7)
        int32_t pages[Loads::kMine], places[Loads::kMine];
#pragma unroll
        for (int n = 0; n < Loads::kMine; ++n) {
            const int r = ((n % Loads::kEach) * 64 + lane) / Loads::kChunks + Loads::kTokens * (n / Loads::kEach);
            pages[n] = __shfl(page, r);
            places[n] = __shfl(place, r);
        }
#pragma unroll
        for (int n = 0; n < Loads::kMine; ++n) {
            const uint32_t e = (uint32_t)(n % Loads::kEach) * 64u + (uint32_t)lane, piece = (e % Loads::kChunks) ^ swizzle<DP>(e / Loads::kChunks);
            const bool there = pages[n] >= 0 && piece * 8u < (uint32_t)a.dim; // (none behind the last key)
            load_to_lds_at(there ? head + (uint64_t)((int64_t)pages[n] * o.batch + (int64_t)places[n] * o.token) + piece * 16u : reinterpret_cast<uint64_t>(kZeros),
                           to + (uint32_t)n * kBlock<DP>);
        }
    }
    __device__ __forceinline__ void load_keys(uint64_t word, uint32_t to) const { load(a.k, k_loads, k_head, word, to); }
    __device__ __forceinline__ void load_values(uint64_t word, uint32_t to) const { load(a.v, v_loads, v_head, word, to); }
};

__device__ __forceinline__ int32_t page_or_none(const Paged &a, int32_t page) { return page >= 0 && page < a.pages ? page : -1; }

// Sixteen rows for each block, in 16 x 16 x 32 instructions: S^T = K Q^T leaves a lane, of row l mod 16 and with g = l / 16, keys 4 g ..
// and 16 + 4 g .. of a tile of 32, which in this order are the second operand of V^T P^T; V^T comes by transposing reads, two for each.
template <class SH> struct PagedRows {
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    static constexpr int DP = SH::DP, BLOCKS = SH::BLOCKS, NS = DP / 32, ND = DP / 16;

    u32x4 q[BLOCKS][NS];   // lane l: row l mod 16, channels 32 s + 8 (l / 16) ..
    f32x4 acc[BLOCKS][ND]; // channels 16 d + 4 (l / 16) ..
    float top[BLOCKS], sum[BLOCKS];
    int32_t last[BLOCKS]; // the last key that the lane's row sees
    int32_t first, seen;  // the least of the rows' last ones; keys that any sees

    __device__ __forceinline__ void load(const Paged &a, int32_t b, int32_t kvh, uint32_t row0, int32_t count, int lane)
    {
        const uint32_t group = (uint32_t)a.group, g = (uint32_t)lane >> 4;
        const uint32_t end = row0 + SH::kRows < (uint32_t)a.rows ? row0 + SH::kRows : (uint32_t)a.rows;
        const int32_t before = count - a.queries;
        first = before + (int32_t)(row0 / group);
        seen = before + (int32_t)((end - 1) / group) + 1;
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n) {
            const uint32_t row = row0 + 16u * n + ((uint32_t)lane & 15u);
            last[n] = before + (int32_t)(row / group);
            const uint64_t at = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head + row_offset(row, group, a.q.token, a.q.head));
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const uint32_t channel = 32u * s + 8u * g;
                q[n][s] = gload16((int64_t)row < a.rows && channel < (uint32_t)a.dim ? at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
                acc[n][d] = f32x4{};
            top[n] = -__builtin_inff();
            sum[n] = 0.0f;
        }
    }

    // The scores of tile t; word: which of its keys there are.
    __device__ __forceinline__ void scores(uint32_t keys_at, int32_t t, uint64_t word, int lane, f32x4 (&x)[BLOCKS][2]) const
    {
        const uint32_t i = (uint32_t)lane & 15u, g = (uint32_t)lane >> 4;
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n)
            x[n][0] = x[n][1] = f32x4{};
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const u32x4 k = lds_read16(keys_at + row_at<DP>(i) + (((uint32_t)(4 * s) + g) ^ swizzle<DP>(i)) * 16u + row_at<DP>(16u * half));
#pragma unroll
                for (int n = 0; n < BLOCKS; ++n)
                    x[n][half] = MM::multiply16(k, q[n][s], x[n][half]);
            }
        if (word != 0xffffffffu || t * kTileKeys + kTileKeys - 1 > first) {
            const uint32_t mine = (uint32_t)word >> (4u * g);
            const int32_t key = t * kTileKeys + 4 * (int32_t)g;
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[n][j / 4][j % 4] = (mine >> (16 * (j / 4) + j % 4) & 1u) && key + 16 * (j / 4) + j % 4 <= last[n] ? x[n][j / 4][j % 4] : -__builtin_inff();
        }
    }
    __device__ __forceinline__ void probabilities(const f32x4 (&x)[BLOCKS][2], float c, u32x4 (&p)[BLOCKS])
    {
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n) {
            float most = x[n][0][0];
#pragma unroll
            for (int j = 1; j < 8; ++j)
                most = fmaxf(most, x[n][j / 4][j % 4]);
            most = quarters_max(most);
            if (__ballot(most > top[n] + fminf(8.0f / c, 1e38f)) != 0) {
                const float next = fmaxf(top[n], most);
                const float by = next > -__builtin_inff() ? __builtin_amdgcn_exp2f((top[n] - next) * c) : 1.0f;
                sum[n] *= by;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    acc[n][d] *= by;
                top[n] = next;
            }
            const float less = top[n] > -__builtin_inff() ? top[n] * c : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float y = __builtin_amdgcn_exp2f(fmaf(x[n][j / 4][j % 4], c, -less)), z = __builtin_amdgcn_exp2f(fmaf(x[n][j / 4][j % 4 + 1], c, -less));
                sum[n] += y + z;
                p[n][j / 2] = MM::two(y, z);
            }
        }
    }
    // channels 16 d .. of the values, as first operand
    static __device__ __forceinline__ u32x4 values(uint32_t values_at, int d, int lane)
    {
        const uint32_t r = (uint32_t)lane >> 2, piece = 2u * d + (((uint32_t)lane & 3u) >> 1);
        const uint32_t at = values_at + row_at<DP>(r) + (piece ^ swizzle<DP>(r)) * 16u + ((uint32_t)lane & 1u) * 8u;
        const u32x2 y = __builtin_bit_cast(u32x2, lds_read_transposed(at)), z = __builtin_bit_cast(u32x2, lds_read_transposed(at + row_at<DP>(16u)));
        u32x4 v;
        v[0] = y[0];
        v[1] = y[1];
        v[2] = z[0];
        v[3] = z[1];
        return v;
    }
    __device__ __forceinline__ void add(const u32x4 (&p)[BLOCKS], uint32_t values_at, int lane)
    {
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const u32x4 v = values(values_at, d, lane);
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n)
                acc[n][d] = MM::multiply16(v, p[n], acc[n][d]);
        }
    }
    // A row at a time, with zeros in place of the values behind its last key (Rows::add_each).
    __device__ __forceinline__ void add_each(const u32x4 (&p)[BLOCKS], uint32_t values_at, int32_t t, int lane)
    {
#pragma unroll 1
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int n = 0; n < BLOCKS; ++n) {
                const int32_t mine = __builtin_amdgcn_readlane(last[n], r) - t * kTileKeys - 4 * (lane >> 4);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    u32x4 v = values(values_at, d, lane);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int32_t key = 16 * (j / 2) + 2 * (j % 2);
                        v[j] = key > mine ? 0u : key + 1 > mine ? v[j] & 0xffffu : v[j];
                    }
                    const f32x4 all = MM::multiply16(v, p[n], acc[n][d]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[n][d][i] = (lane & 15) == r ? all[i] : acc[n][d][i];
                }
            }
    }
    __device__ __forceinline__ bool not_finite() const
    {
        float x = 0.0f;
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x = fmaf(acc[n][d][i], 0.0f, x);
        return __ballot(x != x) != 0;
    }

    // A wavefront's way through tiles t0, t0 + STEP, .. below t1 without a barrier.  Keys and values have a buffer each, and each is loaded
    // anew as soon as it has been read: the next keys are on their way while this tile's probabilities are made, and the other wavefronts'
    // loads while it computes.  Returns whether there was a key.
    template <int STEP> __device__ __forceinline__ bool walk(Pages<SH> &pages, int32_t t0, int32_t t1, uint32_t keys_at, int lane, float c, bool each)
    {
        constexpr int kLoads = TileLoads<DP, kTileKeys, 1>::kMine;
        const uint32_t values_at = keys_at + SH::kTile;
        if (t0 >= t1)
            return false;
        uint64_t word = pages.word(t0), some = word;
        pages.load_keys(word, keys_at);
        pages.load_values(word, values_at);
#pragma unroll 1
        for (int32_t t = t0; t < t1; t += STEP) {
            const bool more = t + STEP < t1;
            wait_loads<kLoads>();
            f32x4 x[BLOCKS][2];
            scores(keys_at, t, word, lane, x);
            const bool some_later = t * kTileKeys + kTileKeys - 1 > first;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (the keys' buffer is loaded into next)
            if (more) {
                word = pages.word(t + STEP);
                some |= word;
                pages.load_keys(word, keys_at);
            }
            u32x4 p[BLOCKS];
            probabilities(x, c, p);
            if (more)
                wait_loads<kLoads>();
            else
                wait_loads<0>();
            if (some_later && each)
                add_each(p, values_at, t, lane);
            else
                add(p, values_at, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more)
                pages.load_values(word, values_at);
        }
        return some != 0;
    }
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int n = 0; n < BLOCKS; ++n)
            arrived(q[n]);
    }
};

// A walk to a workgroup, whose wavefronts share the keys and join what they found.
template <class SH> __global__ __launch_bounds__(64 * kWaves, 2 * SH::kPerUnit) void paged_kernel(const Paged a)
{
    constexpr int DP = SH::DP, KT = kTileKeys, kAll = kWaves * kEntries;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t *const table = reinterpret_cast<int32_t *>(smem + SH::kTable);
    const int32_t units = walks_of(a), b = (int32_t)blockIdx.x / units, unit = (int32_t)blockIdx.x - b * units;
    const int32_t row_tile = unit / a.kv_heads, kvh = unit - row_tile * a.kv_heads;
    const uint32_t row0 = (uint32_t)SH::kRows * (uint32_t)row_tile;
    const int32_t *const entries_of = a.table + (int64_t)b * a.table_stride;
    // (the first entries do not wait for the length)
    const int32_t early = tid < a.entries ? page_or_none(a, entries_of[tid]) : -1;
    const TileLoads<DP, KT, 1> k_loads(0, lane, a.k.token, a.dim), v_loads(0, lane, a.v.token, a.dim);
    PagedRows<SH> rows;
    rows.load(a, b, kvh, row0, keys_of(a, b), lane);
    constexpr int kChunk = (kAll - 1) / KT * KT; // keys, with pages of one
    Pages<SH> pages{a, table, k_loads, v_loads, a.k.at + (uint64_t)(kvh * a.k.head), a.v.at + (uint64_t)(kvh * a.v.head), lane, 0, 0, -1, 0};
    table[tid] = early;
    rows.arrive();
    for (bool each = false;; each = true) {
        rows.clear();
        bool some = false;
#pragma unroll 1
        for (int64_t key0 = 0; key0 < rows.seen; key0 += (int64_t)kChunk * a.page) {
            const int64_t behind = key0 + (int64_t)kChunk * a.page;
            pages.end = behind < rows.seen ? (int32_t)behind : rows.seen;
            pages.first = (int32_t)key0 / a.page;
            const int32_t entries = (pages.end - 1) / a.page - pages.first + 1;
            if (key0 > 0 || each) {
                barrier(); // (all are done with the entries before)
                for (int32_t i = tid; i < entries; i += 64 * kWaves)
                    table[i] = page_or_none(a, entries_of[pages.first + i]);
            } else {
                for (int32_t i = tid + 64 * kWaves; i < entries; i += 64 * kWaves)
                    table[i] = page_or_none(a, entries_of[i]);
            }
            wait_loads<0>();
            barrier();
            some |= rows.template walk<kWaves>(pages, (int32_t)(key0 / KT) + wave, (pages.end + KT - 1) / KT, lds0 + (uint32_t)wave * 2u * SH::kTile, lane, a.c, each);
        }
        if (!some) // (a query may hold NaN, and the scores of keys that are not there are 0 NaN then)
            rows.clear();
        // (all wavefronts, for the barriers; and this one is in front of what is joined, which lies where the tiles were)
        const bool again = __syncthreads_or(rows.not_finite()) != 0;
        if (each || !again)
            break;
    }
    // sums relative to a common maximum, added in wavefront order
    constexpr int kPitch = SH::kPitch, kRows = SH::kRows;
    float *const joined = reinterpret_cast<float *>(smem);     // [wave][row][channel]
    float *const stats = joined + kWaves * kRows * kPitch;     // [wave][2][row]
#pragma unroll
    for (int n = 0; n < SH::BLOCKS; ++n) {
        const int row = 16 * n + (lane & 15);
        const float sum = quarters_sum(rows.sum[n]);
        if (lane < 16) {
            stats[wave * 2 * kRows + row] = rows.top[n];
            stats[wave * 2 * kRows + kRows + row] = sum;
        }
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
            *reinterpret_cast<f32x4 *>(joined + (wave * kRows + row) * kPitch + 16 * d + 4 * (lane >> 4)) = rows.acc[n][d];
    }
    __syncthreads();
    for (int i = tid; i < kRows * (DP / 4); i += 64 * kWaves) {
        const int row = i / (DP / 4), channel = 4 * (i - row * (DP / 4));
        if ((int64_t)row0 + row >= a.rows || channel >= a.dim)
            continue;
        float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            top = fmaxf(top, stats[w * 2 * kRows + row]);
        f32x4 o = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float m = stats[w * 2 * kRows + row], by = m > -__builtin_inff() ? __builtin_amdgcn_exp2f((m - top) * a.c) : 0.0f;
            sum += stats[w * 2 * kRows + kRows + row] * by;
            o += *reinterpret_cast<const f32x4 *>(joined + (w * kRows + row) * kPitch + channel) * by;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        u32x2 w;
        w[0] = Matrix<typename SH::IO>::two(o[0] * inv, o[1] * inv);
        w[1] = Matrix<typename SH::IO>::two(o[2] * inv, o[3] * inv);
        *reinterpret_cast<u32x2 *>(out_row(a, b, kvh, row0 + (uint32_t)row) + 2 * channel) = w;
    }
}

// The walks dealt out evenly to the wavefronts, in groups of 32 keys.  Each goes its way by itself, without a barrier, from walk to walk,
// and leaves what it found of each for the second launch: while one begins or ends a walk, the others' loads keep the memory busy.
// `bundle` wavefronts side by side have the same keys of as many heads, which lie side by side in memory, and count as one worker (a.splits
// of those).
typedef DealOf<Paged, kTileKeys> WaveDeal;
template <class SH> __global__ __launch_bounds__(64 * kWaves, 2 * SH::kPerUnit) void paged_waves_kernel(const Paged a)
{
    constexpr int DP = SH::DP, KT = kTileKeys;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t *const table = reinterpret_cast<int32_t *>(smem + SH::kTable) + wave * kEntries;
    // (the wavefronts of a workgroup are far from one another: the rest of the division is on all compute units)
    const int32_t turn = wave / a.bundle, mine = wave - turn * a.bundle, worker = turn * (int32_t)gridDim.x + (int32_t)blockIdx.x;
    WaveDeal deal(a);
    if (worker >= deal.workers)
        return;
    const TileLoads<DP, KT, 1> k_loads(0, lane, a.k.token, a.dim), v_loads(0, lane, a.v.token, a.dim);
    constexpr int kChunk = (kEntries - 1) / KT * KT; // keys, with pages of one
    int32_t x = deal.first_of(worker);
    const int32_t end = deal.first_of(worker + 1);
    deal.find(a, x);
#pragma unroll 1
    while (x < end) {
        const int32_t unit = (x - deal.begin) / deal.groups, g0 = x - deal.begin - unit * deal.groups, b = deal.b;
        const int32_t g1 = end - x < deal.groups - g0 ? g0 + end - x : deal.groups;
        const int32_t walk = unit * a.bundle + mine, row_tile = walk / a.kv_heads, kvh = walk - row_tile * a.kv_heads;
        const uint32_t row0 = (uint32_t)SH::kRows * (uint32_t)row_tile;
        PagedRows<SH> rows;
        rows.load(a, b, kvh, row0, deal.count, lane);
        const int32_t stop = g1 * KT < rows.seen ? g1 * KT : rows.seen;
        const int32_t *const entries_of = a.table + (int64_t)b * a.table_stride;
        Pages<SH> pages{a, table, k_loads, v_loads, a.k.at + (uint64_t)(kvh * a.k.head), a.v.at + (uint64_t)(kvh * a.v.head), lane, 0, 0, -1, 0};
#pragma unroll 1
        for (bool each = false;; each = true) {
            rows.clear();
            bool some = false;
#pragma unroll 1
            for (int64_t key0 = (int64_t)g0 * KT; key0 < stop; key0 += (int64_t)kChunk * a.page) {
                const int64_t behind = key0 + (int64_t)kChunk * a.page;
                pages.end = behind < stop ? (int32_t)behind : stop;
                pages.first = (int32_t)key0 / a.page;
                const int32_t entries = (pages.end - 1) / a.page - pages.first + 1;
                for (int32_t i = lane; i < entries; i += 64)
                    table[i] = page_or_none(a, entries_of[pages.first + i]);
                rows.arrive();
                wait_loads<0>();
                some |= rows.template walk<1>(pages, (int32_t)(key0 / KT), (pages.end + KT - 1) / KT, lds0 + (uint32_t)wave * 2u * SH::kTile, lane, a.c, each);
            }
            if (!some) // (a query may hold NaN, and the scores of keys that are not there are 0 NaN then)
                rows.clear();
            if (each || !rows.not_finite())
                break;
        }
        const int64_t slot = ((int64_t)b * units_of(a) + unit + worker) * a.bundle + mine;
#pragma unroll
        for (int n = 0; n < SH::BLOCKS; ++n) {
            const float sum = quarters_sum(rows.sum[n]), inv = sum == 0.0f ? 0.0f : 1.0f / sum, l2 = log2_sum(rows.top[n], sum, a.c);
            const int32_t row = 16 * n + (lane & 15);
            if ((int64_t)row0 + row >= a.rows)
                continue;
            float *const out = a.partial + (slot * a.unit_rows + row) * a.dim;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
                if (const int channel = 16 * d + 4 * (lane >> 4); channel < a.dim)
                    *reinterpret_cast<f32x4 *>(out + channel) = rows.acc[n][d] * inv;
            if (lane < 16)
                a.partial[slots_of(a) * a.unit_rows * a.dim + slot * a.unit_rows + row] = l2;
        }
        x += g1 - g0;
        if (x < end && x == deal.begin + deal.groups * units_of(a)) { // the next sequence with keys
            deal.begin = x;
            do {
                deal.count = keys_of(a, ++deal.b);
                deal.groups = WaveDeal::groups_of(deal.count);
            } while (deal.groups == 0);
        }
    }
}

// out of the workers' parts: a.join_lanes lanes for eight channels of a row
template <typename IO> __global__ __launch_bounds__(256) void join_paged_kernel(const Paged a)
{
    const uint32_t pieces = (uint32_t)a.dim / 8u, lanes = (uint32_t)a.join_lanes, all = (uint32_t)a.unit_rows * pieces, each = 256u / lanes;
    const int32_t turns = (int32_t)((all + each - 1) / each), place = (int32_t)blockIdx.x / turns, turn = (int32_t)blockIdx.x - place * turns;
    const int32_t walks = walks_of(a), b = place / walks, walk = place - b * walks, unit = walk / a.bundle, mine = walk - unit * a.bundle;
    const int32_t row_tile = walk / a.kv_heads, kvh = walk - row_tile * a.kv_heads;
    WaveDeal deal(a);
    deal.find(a, -1, b);
    const int32_t x0 = deal.begin + unit * deal.groups;
    const int32_t w0 = deal.groups ? deal.worker_of(x0) : 0, parts = deal.groups ? deal.worker_of(x0 + deal.groups - 1) - w0 + 1 : 0;
    const uint32_t sub = threadIdx.x & (lanes - 1), item = (uint32_t)turn * each + threadIdx.x / lanes, row = item / pieces, piece = item - row * pieces;
    const uint32_t row_at = (uint32_t)(a.tile_rows * row_tile) + row;
    if (item >= all || (int64_t)row_at >= a.rows)
        return;
    const float *const stats = a.partial + slots_of(a) * a.unit_rows * a.dim;
    const int64_t first = (int64_t)b * units_of(a) + unit + w0;
    auto line = [&](int32_t p) { return ((first + p) * a.bundle + mine) * a.unit_rows + row; };
    join_parts<IO>(
        parts, (int32_t)sub, (int32_t)lanes, [&](int32_t p) { return a.partial + line(p) * a.dim + 8u * piece; }, [&](int32_t p) { return stats[line(p)]; },
        out_row(a, b, kvh, row_at) + 16u * piece);
}

// ------------------------------------------------------------------------------------------------ into the pages

constexpr int kMostTokens = 64; // a lane of a wavefront each

struct PagedWrite : Packed { // k, v: of the new tokens; rows: tokens
    char *k_pages, *v_pages;
    int64_t k_page, k_place, k_place_head, v_page, v_place, v_place_head; // bytes
    const int32_t *table;
    const void *lengths;
    int64_t table_stride, pages;
    int32_t lengths_64, page, entries;
    int32_t per; // tokens of a workgroup, kMostTokens at most
};

// A copy, 16 bytes a lane: bound by memory, or for few tokens by the way from the offsets over the lengths and the table to the page.
__global__ __launch_bounds__(256) void paged_write_kernel(const PagedWrite a)
{
    __shared__ int32_t page_of[kMostTokens], place_of[kMostTokens];
    const int32_t token0 = (int32_t)blockIdx.x * a.per, here = a.tokens - token0 < a.per ? a.tokens - token0 : a.per;
    if (threadIdx.x < kMostTokens) {
        const int32_t lane = (int32_t)threadIdx.x, token = token0 + lane;
        // the segment of the workgroup's first token: the last that begins at or in front of it
        int32_t lo = 0, len = a.sequences + 2;
        while (len > 1) {
            const int32_t step = (len + 63) / 64, i = lo + lane * step;
            const uint64_t found = __ballot(lane * step < len && boundary(a, i) <= token0) | 1u;
            const int32_t j = 63 - __builtin_clzll(found);
            lo += j * step;
            len = len - j * step < step ? len - j * step : step;
        }
        // of the others: 64 boundaries at a time
        int32_t segment = lo, begin = 0, end = 0;
        for (int32_t base = lo;; base += 63) {
            const int32_t mine = boundary(a, base + lane);
            for (int32_t i = 0; i < 63; ++i) {
                const int32_t b0 = __builtin_amdgcn_readlane(mine, i), b1 = __builtin_amdgcn_readlane(mine, i + 1);
                const bool in = token >= b0 && token < b1;
                segment = in ? base + i : segment;
                begin = in ? b0 : begin;
                end = in ? b1 : end;
            }
            if (base + 63 >= a.sequences + 2 || __builtin_amdgcn_readlane(mine, 63) > token0 + here - 1)
                break;
        }
        int32_t page = -1, place = 0;
        if (lane < here && token >= begin && token < end && segment >= 1 && segment <= a.sequences) {
            const int32_t s = segment - 1;
            const int64_t length = a.lengths_64 ? static_cast<const int64_t *>(a.lengths)[s] : (int64_t) static_cast<const int32_t *>(a.lengths)[s];
            const int64_t position = length - (end - token);
            if (length <= a.keys && position >= 0) {
                const int32_t entry = (int32_t)position / a.page;
                page = a.table[(int64_t)s * a.table_stride + entry];
                place = (int32_t)position - entry * a.page;
                page = page >= 0 && page < a.pages ? page : -1;
            }
        }
        page_of[lane] = page;
        place_of[lane] = place;
    }
    __syncthreads();
    const uint32_t chunks = (uint32_t)a.dim / 8u, pieces = chunks * (uint32_t)a.kv_heads, items = (uint32_t)here * pieces;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += 4 * 256) {
        u32x4 k[4], v[4];
        uint64_t k_to[4], v_to[4];
        bool there[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t given = i0 + 256u * n, i = given < items ? given : items - 1;
            const uint32_t token = i / pieces, piece = i - token * pieces, head = piece / chunks, chunk = piece - head * chunks;
            const int64_t page = page_of[token], place = place_of[token];
            there[n] = given < items && page >= 0;
            const int64_t t = (int64_t)token0 + token;
            k[n] = gload16(a.k.at + (uint64_t)(t * a.k.token + head * a.k.head) + 16u * chunk, 0);
            v[n] = gload16(a.v.at + (uint64_t)(t * a.v.token + head * a.v.head) + 16u * chunk, 0);
            k_to[n] = reinterpret_cast<uint64_t>(a.k_pages) + (uint64_t)(page * a.k_page + place * a.k_place + head * a.k_place_head) + 16u * chunk;
            v_to[n] = reinterpret_cast<uint64_t>(a.v_pages) + (uint64_t)(page * a.v_page + place * a.v_place + head * a.v_place_head) + 16u * chunk;
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (there[n]) {
                gstore16(k_to[n], 0, k[n]);
                gstore16(v_to[n], 0, v[n]);
            }
    }
}

// ------------------------------------------------------------------------------------------------ host

static grkan_status_t check_cache(const grkan_paged_cache_t *c, grkan_dtype_t io)
{
    if (!c)
        return GRKAN_ERR_NULL;
    if (c->pages < 0 || c->page_size < 1 || c->sequences < 0 || c->table_entries < 0 || c->kv_heads < 1 || c->dim < 1)
        return GRKAN_ERR_SHAPE;
    if (io != GRKAN_BF16 && io != GRKAN_F16)
        return GRKAN_ERR_DTYPE;
    const int64_t most = (int64_t)1 << 30;
    if (c->dim % 8 != 0 || c->dim > 128 || c->pages >= (int64_t)1 << 31 || (int64_t)c->page_size * c->table_entries >= most || c->page_size >= most)
        return GRKAN_ERR_UNSUPPORTED;
    if (!in_offsets(c->k_token_stride, 0, 1) || !in_offsets(c->v_token_stride, 0, 1))
        return GRKAN_ERR_UNSUPPORTED;
    if (c->sequences > 0 && (!c->lengths || (c->table_entries > 0 && !c->table) || (c->pages > 0 && (!c->k_pages || !c->v_pages))))
        return GRKAN_ERR_NULL;
    auto address = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if ((address(c->k_pages) | address(c->v_pages)) % 16 != 0 || address(c->table) % 4 != 0 || address(c->lengths) % (c->lengths_64 ? 8 : 4) != 0 ||
        (c->k_page_stride | c->k_token_stride | c->k_head_stride | c->v_page_stride | c->v_token_stride | c->v_head_stride) % 8 != 0)
        return GRKAN_ERR_ALIGN;
    return GRKAN_OK;
}

static grkan_status_t fill(const grkan_paged_cache_t *c, const grkan_paged_queries_t *q, grkan_dtype_t io, Paged *to)
{
    if (!q)
        return GRKAN_ERR_NULL;
    const grkan_status_t bad = check_cache(c, io);
    if (bad != GRKAN_OK)
        return bad;
    if (q->tokens < 0 || q->heads < 1 || q->heads % c->kv_heads != 0)
        return GRKAN_ERR_SHAPE;
    const int64_t group = q->heads / c->kv_heads, rows = q->tokens * group;
    if (!(q->scale > 0) || !std::isfinite(q->scale * 1.4426950408889634f))
        return GRKAN_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)1 << 30;
    if (q->tokens >= most || rows >= most || (rows + 15) / 16 * c->kv_heads >= most)
        return GRKAN_ERR_UNSUPPORTED;
    if (c->sequences > 0 && rows > 0 && !q->q)
        return GRKAN_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(q->q) % 16 != 0 || (q->sequence_stride | q->token_stride | q->head_stride) % 8 != 0)
        return GRKAN_ERR_ALIGN;
    Paged a = {};
    a.q = Operand{reinterpret_cast<uint64_t>(q->q), q->sequence_stride * 2, q->token_stride * 2, q->head_stride * 2};
    a.k = Operand{reinterpret_cast<uint64_t>(c->k_pages), c->k_page_stride * 2, c->k_token_stride * 2, c->k_head_stride * 2};
    a.v = Operand{reinterpret_cast<uint64_t>(c->v_pages), c->v_page_stride * 2, c->v_token_stride * 2, c->v_head_stride * 2};
    a.lengths = c->lengths;
    a.lengths_64 = c->lengths_64;
    a.keys = (int64_t)c->page_size * c->table_entries;
    a.rows = rows;
    a.batch = c->sequences;
    a.kv_heads = c->kv_heads;
    a.group = (int32_t)group;
    a.dim = c->dim;
    a.scale = q->scale;
    a.c = q->scale * 1.4426950408889634f;
    a.table = c->table;
    a.table_stride = c->table_stride;
    a.pages = c->pages;
    a.page = c->page_size;
    a.entries = c->table_entries;
    a.queries = (int32_t)q->tokens;
    a.tile_rows = rows <= 16 ? 16 : 32;
    a.row_tiles = (int32_t)((rows + a.tile_rows - 1) / a.tile_rows);
    a.unit_rows = rows < a.tile_rows ? (int32_t)rows : a.tile_rows;
    // As many wavefronts as the device holds, or one for each tile of 32 keys; none where a workgroup for each walk does as well: 1,024 of
    // them, or all short, as the second launch takes 4 to 8 us.  us of a call without and with, one walk to each of twelve heads of 64
    // channels: 1,300 keys 9.7 / 12.4, 2,000 12.3 / 12.6, 3,000 16.1 / 13.4; 192 of them 1,500 12.1 / 18.5; 768 1,300 34.7 / 38.9.  Eight
    // of 128 channels: 1,000 11.5 / 13.9, 1,400 13.0 / 14.8, 2,000 16.8 / 14.1, on pages of 16 1,400 17.9 / 15.3; 128 of them 2,000 20.4 /
    // 23.6, 3,000 34.5 / 28.2.
    const int64_t walks = (int64_t)a.batch * a.kv_heads * a.row_tiles, groups = (a.keys + 31) / 32;
    a.bundle = 1;
    a.splits = 0;
    const int64_t alone = a.dim <= 64 || (a.page % 32 == 0 && walks >= 64) ? 64 : a.page % 32 == 0 ? 48 : 40; // groups of a workgroup
    if (walks > 0 && walks < 1024 && groups > alone && walks * groups < most) {
        while (a.bundle < kWaves && a.kv_heads * a.row_tiles % (2 * a.bundle) == 0)
            a.bundle *= 2;
        const int64_t waves = a.dim > 64 ? 2048 : 4096, blocks = ((walks * groups < waves ? walks * groups : waves) + kWaves - 1) / kWaves;
        a.splits = (int32_t)(blocks * kWaves / a.bundle);
        const int32_t each = (int32_t)((int64_t)a.splits * a.bundle / walks) + 1; // parts of a walk
        a.join_lanes = 1;
        while (a.join_lanes < 64 && a.join_lanes * 4 < each)
            a.join_lanes *= 2;
    }
    *to = a;
    return GRKAN_OK;
}

static size_t workspace_of(const Paged &a)
{
    return a.splits > 0 ? ((size_t)a.batch * (size_t)a.kv_heads * (size_t)a.row_tiles + (size_t)a.splits * (size_t)a.bundle) * (size_t)a.unit_rows * (size_t)(a.dim + 1) * sizeof(float)
                        : 0;
}

typedef void (*Kernel)(Paged);
struct PagedVariant {
    Kernel kernel, waves, join;
    size_t lds;
};
template <typename IO, int DP, int BLOCKS> static PagedVariant variant()
{
    using SH = PagedShape<IO, DP, BLOCKS>;
    return PagedVariant{paged_kernel<SH>, paged_waves_kernel<SH>, join_paged_kernel<IO>, SH::kLds};
}
template <typename IO, int DP> static PagedVariant variant(int32_t rows) { return rows <= 16 ? variant<IO, DP, 1>() : variant<IO, DP, 2>(); }
template <typename IO> static PagedVariant pick(int32_t dim, int32_t rows)
{
    return dim <= 32 ? variant<IO, 32>(rows) : dim <= 64 ? variant<IO, 64>(rows) : dim <= 96 ? variant<IO, 96>(rows) : variant<IO, 128>(rows);
}

} // namespace attention
} // namespace grkan

using namespace grkan;

extern "C" size_t grkan_paged_attention_workspace_bytes(const grkan_paged_cache_t *cache, const grkan_paged_queries_t *queries)
{
    attention::Paged a;
    return attention::fill(cache, queries, GRKAN_BF16, &a) == GRKAN_OK ? attention::workspace_of(a) : 0;
}

extern "C" grkan_status_t grkan_paged_attention(const grkan_paged_cache_t *cache, const grkan_paged_queries_t *queries, void *out, void *workspace,
                                                size_t workspace_bytes, grkan_dtype_t io, void *hip_stream)
{
    attention::Paged a;
    const grkan_status_t bad = attention::fill(cache, queries, io, &a);
    if (bad != GRKAN_OK)
        return bad;
    if ((int64_t)a.batch * a.rows == 0)
        return GRKAN_OK;
    if (!out)
        return GRKAN_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(out) % 16 != 0)
        return GRKAN_ERR_ALIGN;
    const size_t need = attention::workspace_of(a);
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
        return GRKAN_ERR_WORKSPACE;
    const int64_t walks = (int64_t)a.batch * a.kv_heads * a.row_tiles, work = a.splits > 0 ? (int64_t)a.splits * a.bundle / attention::kWaves : walks;
    const int64_t each = need ? 256 / a.join_lanes : 1, join = need ? walks * ((a.unit_rows * (a.dim / 8) + each - 1) / each) : 0;
    if (work > attention::kMostBlocks * 4 / attention::kWaves) // (the second launch's are far fewer)
        return GRKAN_ERR_UNSUPPORTED;
    a.out = static_cast<char *>(out);
    a.partial = static_cast<float *>(workspace);
    const attention::PagedVariant v = io == GRKAN_BF16 ? attention::pick<__bf16>(a.dim, a.tile_rows) : attention::pick<_Float16>(a.dim, a.tile_rows);
    const void *const kernel = reinterpret_cast<const void *>(need ? v.waves : v.kernel);
    if (!attention::allow_lds(kernel, v.lds))
        return GRKAN_ERR_LAUNCH;
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    void *args[] = {&a};
    if (hipLaunchKernel(kernel, dim3((unsigned)work), dim3(64 * attention::kWaves), args, v.lds, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    if (need && hipLaunchKernel(reinterpret_cast<const void *>(v.join), dim3((unsigned)join), dim3(256), args, 0, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    return GRKAN_OK;
}

extern "C" grkan_status_t grkan_paged_write(const grkan_paged_cache_t *cache, const void *k, const void *v, const void *offsets, int32_t offsets_64,
                                            int64_t tokens, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                                            grkan_dtype_t io, void *hip_stream)
{
    const grkan_status_t bad = attention::check_cache(cache, io);
    if (bad != GRKAN_OK)
        return bad;
    if (tokens < 0 || (!offsets && (cache->sequences == 0 ? tokens != 0 : tokens % cache->sequences != 0)))
        return GRKAN_ERR_SHAPE;
    if (tokens > attention::kMostTokens * attention::kMostBlocks || (int64_t)cache->kv_heads * cache->dim >= (int64_t)1 << 24 || cache->sequences >= 1 << 30)
        return GRKAN_ERR_UNSUPPORTED;
    if (tokens == 0 || cache->sequences == 0 || cache->pages == 0)
        return GRKAN_OK;
    if (!k || !v)
        return GRKAN_ERR_NULL;
    auto address = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if ((address(k) | address(v)) % 16 != 0 || address(offsets) % (offsets_64 ? 8 : 4) != 0 || (k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8 != 0)
        return GRKAN_ERR_ALIGN;
    attention::PagedWrite a = {};
    a.k = attention::Operand{address(k), 0, k_token_stride * 2, k_head_stride * 2};
    a.v = attention::Operand{address(v), 0, v_token_stride * 2, v_head_stride * 2};
    a.kv_heads = cache->kv_heads;
    a.dim = cache->dim;
    a.offsets = offsets;
    a.offsets_64 = offsets_64;
    a.sequences = cache->sequences;
    a.tokens = (int32_t)tokens;
    a.each = (int32_t)(tokens / cache->sequences);
    a.keys = (int64_t)cache->page_size * cache->table_entries;
    a.k_pages = static_cast<char *>(cache->k_pages);
    a.v_pages = static_cast<char *>(cache->v_pages);
    a.k_page = cache->k_page_stride * 2;
    a.k_place = cache->k_token_stride * 2;
    a.k_place_head = cache->k_head_stride * 2;
    a.v_page = cache->v_page_stride * 2;
    a.v_place = cache->v_token_stride * 2;
    a.v_place_head = cache->v_head_stride * 2;
    a.table = cache->table;
    a.lengths = cache->lengths;
    a.lengths_64 = cache->lengths_64;
    a.table_stride = cache->table_stride;
    a.pages = cache->pages;
    a.page = cache->page_size;
    a.entries = cache->table_entries;
    const int64_t per = (tokens + 1023) / 1024;
    a.per = (int32_t)(per < attention::kMostTokens ? per : attention::kMostTokens);
    const int64_t grid = (tokens + a.per - 1) / a.per;
    attention::paged_write_kernel<<<dim3((unsigned)grid), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(a);
    return hipGetLastError() == hipSuccess ? GRKAN_OK : GRKAN_ERR_LAUNCH;
}
