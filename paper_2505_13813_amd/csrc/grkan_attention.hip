// Cross attention on gfx950 (MI355X), forward: out = softmax(scale Q K^T) V in one pass over the keys, with the running maximum and sum
// of each row.
//
//   * With rows enough (queries x heads that share a key head), a workgroup of four wavefronts has 32 each; 64 keys and their
//     values at a time come to LDS by LDS-direct loads, two tiles deep, and serve all four.
//     Where the workgroups would not fill the chip, the keys are split over several, and a second launch joins them.
//   * With 32 rows or fewer (single tokens), or few tiles of 32, the keys are what there is to read: the four wavefronts have the same rows and
//     tiles of 32 keys of their own, in LDS of their own, without a barrier, and join what they found at the end.  Where single tokens' keys are long, they are dealt
//     out evenly to a workgroup on each compute unit, and a second launch joins the parts.
//
// What bounds them.  Many rows: 4 dim products and some 1.3 vector operations and an exponential for each score, and little of the two runs
// at once: a loop of these alone, without memory, takes 510 ns for 32 rows, 64 keys and 64 channels with three wavefronts on a SIMD, its products alone
// 245; here it is 655 with four (16 x 2048 x 2048 of 12 heads: 252 us = 820 TFLOP/s; 4 x 2048 x 2048 of 16 heads of 128 165 us = 830; 2 x 4096 queries, 4,001 and 1,808 keys of 16
// heads of 128: 219 us = 890).  Few rows: memory (16 single tokens of 32 heads, 2,268 to 8,191 keys of eight, 0.29 GB: 62 us = 4.6 TB/s, and 5 to join).
//
// The maximum of a row is raised only where a score passes it by more than 2^8 in the exponent: the probabilities are then at most 256,
// which neither 16-bit type minds, and the accumulators are scaled in few of the tiles instead of in most.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <unordered_set>

#include "grkan_attention_rows.h"

namespace grkan {
namespace attention {

// ------------------------------------------------------------------------------------------------ many rows

template <typename IO_, int DP_> struct Shape {
    typedef IO_ IO;
    static constexpr int DP = DP_, KT = 64, kWaves = 4, kRows = 32 * kWaves;
    static constexpr uint32_t kTile = kTileBytes<DP, KT>;
    static constexpr uint32_t kCover = 4 * kTile; // behind K and V, two of each
    static constexpr size_t kLds = kCover + 2 * KT * 4;
};

// Up to 64 channels four workgroups fit a compute unit (128 registers; us with three, of 129, and with four: 16 x 2048 x 2048 of 12 heads of 64
// 266 to 289 / 252, 4 x 2048 x 2048 of 16 115 to 124 / 110, 64 x 197 x 360 of 12 38 / 37, and 32 x 256 x 785 of 12, which is one round of three, 36 / 37).
template <class SH> __global__ __launch_bounds__(256, SH::DP <= 64 ? 4 : 2) void forward_kernel(const Args a)
{
    constexpr int DP = SH::DP, KT = SH::KT;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;

    const int32_t item = work_item(a);
    if (item >= a.work)
        return;
    const int32_t per_head = a.row_tiles * a.splits;
    const int32_t bh = item / per_head, rest = item - bh * per_head;
    const int32_t row_tile = rest / a.splits, split = rest - row_tile * a.splits;
    const int32_t b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    const uint32_t row0 = (uint32_t)row_tile * SH::kRows + (uint32_t)wave * 32u, row = row0 + col;
    Rows<typename SH::IO, DP, KT> rows;
    rows.load(a, b, kvh, row, h);
    rows.clear();

    const int32_t count = keys_of(a, b), tiles = (count + KT - 1) / KT;
    int32_t t0 = split * a.tiles_per_split, t1 = t0 + a.tiles_per_split;
    t1 = t1 < tiles ? t1 : tiles;
    const TileLoads<DP, KT, SH::kWaves> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    const RowOperand<DP> k_operand(lane);
    const ColumnOperand<DP> v_operand(lane);
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
    ValidKeys valid(a, b, count, t1);
    auto issue = [&](int32_t t, uint64_t word, uint32_t at) {
        const bool all = word == ~(uint64_t)0, whole = all && a.dim == DP;
        k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, a.k.token, word, whole, lds0 + at);
        v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, a.v.token, word, whole, lds0 + at + 2 * SH::kTile);
        if (!all && wave == 0)
            write_cover(lds0 + SH::kCover + (at ? KT * 4u : 0u), word, lane);
    };
    arrived(rows.q);
    uint64_t some = 0; // valid keys
    // (a wavefront without rows loads for the others; two loops, as one with a condition in it would copy the sums in every pass)
    auto walk = [&](auto works) {
        uint32_t at = 0;
        uint64_t word = 0;
        if (t0 < t1) {
            word = valid.word(t0);
            issue(t0, word, 0);
        }
        for (int32_t t = t0; t < t1; ++t) {
            const uint64_t next = t + 1 < t1 ? valid.word(t + 1) : 0;
            wait_loads<0>();
            barrier(); // all wavefronts' loads of this tile are there, and all are done with the tile before
            if (t + 1 < t1)
                issue(t + 1, next, at ^ SH::kTile);
            if constexpr (decltype(works)::value)
                rows.take(k_operand.moved(lds0 + at), v_operand.moved(lds0 + at + 2 * SH::kTile), word,
                          lds0 + SH::kCover + (at ? KT * 4u : 0u), a.c, h);
            at ^= SH::kTile;
            some |= word;
            word = next;
        }
    };
    if ((int64_t)row0 >= a.rows) {
        walk(std::false_type{});
        return;
    }
    walk(std::true_type{});
    if (some == 0) // (a query may hold NaN, and masked keys' scores are 0 NaN then)
        rows.clear();
    if ((int64_t)row >= a.rows)
        return;

    const float sum = halves_sum(rows.sum), inv = sum == 0.0f ? 0.0f : 1.0f / sum, l2 = log2_sum(rows.top, sum, a.c);
    const bool wide = a.splits > 1;
    const int64_t line = ((int64_t)split * a.batch * a.kv_heads + bh) * a.rows + row;
    char *const out = wide ? reinterpret_cast<char *>(a.partial + line * a.dim) : out_row(a, b, kvh, row);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
        store_channels<typename SH::IO>(rows.acc[d], d, inv, a, out, wide, h);
    if (h == 0) {
        if (wide)
            a.partial[(int64_t)a.splits * a.batch * a.kv_heads * a.rows * a.dim + line] = l2;
        else if (a.lse)
            a.lse[line] = lse_of(l2);
    }
}

// out of the splits' rows: dim / 8 lanes a row
template <typename IO> __global__ __launch_bounds__(256) void join_kernel(const Args a)
{
    const int64_t all = (int64_t)a.batch * a.kv_heads * a.rows;
    const uint32_t pieces = (uint32_t)a.dim / 8u;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, line = i / pieces;
    const uint32_t piece = (uint32_t)(i - line * pieces);
    if (line >= all)
        return;
    const float *const stats = a.partial + (int64_t)a.splits * all * a.dim;
    const int64_t bh = line / a.rows;
    const int32_t b = (int32_t)(bh / a.kv_heads), kvh = (int32_t)(bh - (int64_t)b * a.kv_heads);
    const float lse = join_parts<IO>(
        a.splits, 0, 1, [&](int32_t p) { return a.partial + (p * all + line) * a.dim + 8u * piece; }, [&](int32_t p) { return stats[p * all + line]; },
        out_row(a, b, kvh, (uint32_t)(line - bh * a.rows)) + 16u * piece);
    if (a.lse && piece == 0)
        a.lse[line] = lse;
}

// ------------------------------------------------------------------------------------------------ few rows

// Worker w of W has groups w G / W .. (w + 1) G / W, G all of them (Deal): all have the same to read.  A worker's part of key head bh is in slot bh + w of the workspace (no two are
// in the same: from one part to the next, bh or w rises).
constexpr int kWorkers = 256;

// With a.splits workers (32 rows at most); 0: each has 32 rows of one key head by itself and writes the output.
template <class SH> __global__ __launch_bounds__(256, SH::DP > 64 ? 1 : 2) void tokens_kernel(const Args a)
{
    constexpr int DP = SH::DP, KT = SH::KT;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t row = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    const bool shared = a.splits > 0;
    const int32_t worker = (int32_t)blockIdx.x;

    const TileLoads<DP, KT, 1> k_loads(0, lane, a.k.token, a.dim), v_loads(0, lane, a.v.token, a.dim);

    // rows row0 .. row0 + 31 and groups [g0, g1) of a key head
    auto part = [&](int32_t b, int32_t kvh, uint32_t row0, int32_t count, int32_t g0, int32_t g1) {
        Rows<typename SH::IO, DP, KT> rows;
        rows.load(a, b, kvh, row0 + row, h);
        rows.clear();
        constexpr int kTiles = kGroup / KT;
        const int32_t tiles = (count + KT - 1) / KT, t0 = g0 * kTiles + wave, t1 = g1 * kTiles < tiles ? g1 * kTiles : tiles;
        const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
        ValidKeys valid(a, b, count, (t1 * KT + 63) / 64);
        const bool some = walk_alone<SH>(
            rows, t0, t1, lds0, wave, lane, a.c, a.dim, [&](int32_t t) { return (valid.word(t / 2) >> (t % 2 * 32)) & rows.kAll; },
            [&](int32_t t, uint64_t word, bool whole, uint32_t to) {
                k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, a.k.token, word, whole, to);
                v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, a.v.token, word, whole, to + SH::kTile);
            });
        if (!some) // (a query may hold NaN, and masked keys' scores are 0 NaN then)
            rows.clear();
        const int64_t bh = (int64_t)b * a.kv_heads + kvh, slot = bh + worker;
        char *const out = shared ? reinterpret_cast<char *>(a.partial + (slot * a.rows + row) * a.dim) : out_row(a, b, kvh, row0 + row);
        float *const lse = shared ? a.partial + ((int64_t)a.batch * a.kv_heads + a.splits) * a.rows * a.dim + slot * a.rows + row
                                  : a.lse + (a.lse ? bh * a.rows + row0 + row : 0);
        join_wavefronts<SH>(rows, smem, wave, lane, (int64_t)row0 + row < a.rows, a, out, lse, shared);
    };

    if (!shared) {
        const int32_t bh = worker / a.row_tiles, b = bh / a.kv_heads, count = keys_of(a, b);
        part(b, bh - b * a.kv_heads, 32u * (uint32_t)(worker - bh * a.row_tiles), count, 0, Deal::groups_of(count));
        return;
    }
    Deal deal(a);
    if (worker >= deal.workers)
        return;
    int32_t x = deal.first_of(worker);
    const int32_t end = deal.first_of(worker + 1);
    deal.find(a, x);
    while (x < end) {
        const int32_t kvh = (x - deal.begin) / deal.groups, g0 = x - deal.begin - kvh * deal.groups;
        const int32_t g1 = end - x < deal.groups - g0 ? g0 + end - x : deal.groups;
        part(deal.b, kvh, 0, deal.count, g0, g1);
        x += g1 - g0;
        if (x < end && x == deal.begin + deal.groups * a.kv_heads) { // the next entry with keys
            deal.begin = x;
            do {
                deal.count = keys_of(a, ++deal.b);
                deal.groups = Deal::groups_of(deal.count);
            } while (deal.groups == 0);
        }
    }
}

// out of the workers' parts: a workgroup for each key head, dim / 8 lanes a row, or sixteen times as many at most where the rows leave lanes over
template <typename IO> __global__ __launch_bounds__(256) void join_tokens_kernel(const Args a)
{
    const int32_t bh = (int32_t)blockIdx.x, b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    Deal deal(a);
    deal.find(a, -1, b);
    const int32_t x0 = deal.begin + kvh * deal.groups;
    const int32_t w0 = deal.groups ? deal.worker_of(x0) : 0, parts = deal.groups ? deal.worker_of(x0 + deal.groups - 1) - w0 + 1 : 0;
    const uint32_t pieces = (uint32_t)a.dim / 8u;
    const float *const stats = a.partial + ((int64_t)a.batch * a.kv_heads + a.splits) * a.rows * a.dim;
    const uint32_t items = (uint32_t)a.rows * pieces;
    uint32_t lanes = 1;
    while (lanes < 16 && items * lanes * 2 <= 256)
        lanes *= 2;
    const uint32_t sub = threadIdx.x & (lanes - 1);
    for (uint32_t i = threadIdx.x / lanes; i < items; i += 256 / lanes) {
        const uint32_t row = i / pieces, piece = i - row * pieces;
        auto line = [&](int32_t p) { return ((int64_t)bh + w0 + p) * a.rows + row; };
        const float lse = join_parts<IO>(
            parts, (int32_t)sub, (int32_t)lanes, [&](int32_t p) { return a.partial + line(p) * a.dim + 8u * piece; }, [&](int32_t p) { return stats[line(p)]; },
            out_row(a, b, kvh, row) + 16u * piece);
        if (a.lse && piece == 0 && sub == 0)
            a.lse[(int64_t)bh * a.rows + row] = lse;
    }
}

// ------------------------------------------------------------------------------------------------ host

bool allow_lds(const void *kernel, size_t bytes)
{
    if (bytes <= 64 * 1024)
        return true;
    static std::mutex mu;
    static std::unordered_set<const void *> done[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return false;
    try { // (no exception leaves the C interface)
        std::lock_guard<std::mutex> lock(mu);
        if (done[dev].count(kernel))
            return true;
        if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
            return false;
        done[dev].insert(kernel);
    } catch (...) {
        return false;
    }
    return true;
}

int64_t spread(Args &a, int64_t work, int64_t per_head)
{
    int64_t run = work / 64 < per_head ? work / 64 : per_head;
    run = run > 1 ? run : 1;
    a.work = (int32_t)work;
    a.run = (int32_t)run;
    return (work + 8 * run - 1) / (8 * run) * 8 * run;
}

static bool fine_operand(const void *p, int64_t batch, int64_t token, int64_t head)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (batch | token | head) % 8 == 0;
}

bool in_offsets(int64_t token_stride, int64_t head_stride, int64_t heads)
{
    // 64 tokens and the heads of a group, in bytes, in 32 bits
    const int64_t most = (int64_t)1 << 30;
    return token_stride >= 0 && head_stride >= 0 && token_stride <= (most - 256) / 64 && head_stride <= (most - 256) / heads;
}

grkan_status_t fill(const grkan_attention_t *at, grkan_dtype_t io, Args *to)
{
    if (!at)
        return GRKAN_ERR_NULL;
    if (at->batch < 0 || at->queries < 0 || at->keys < 0 || at->heads < 1 || at->kv_heads < 1 || at->heads % at->kv_heads != 0 || at->dim < 1)
        return GRKAN_ERR_SHAPE;
    if (io != GRKAN_BF16 && io != GRKAN_F16)
        return GRKAN_ERR_DTYPE;
    const int64_t group = at->heads / at->kv_heads;
    if (at->dim % 8 != 0 || at->dim > 128 || !(at->scale > 0) || !std::isfinite(at->scale * 1.4426950408889634f))
        return GRKAN_ERR_UNSUPPORTED;
    // rows and tiles are counted in 31 bits, offsets in a tile of 64 tokens too
    const int64_t most = (int64_t)1 << 31;
    if (at->batch >= most || at->keys > most - 256 || at->queries >= most || at->queries * group >= most - 256 || at->batch * at->kv_heads >= most)
        return GRKAN_ERR_UNSUPPORTED;
    if (!in_offsets(at->k_token_stride, 0, 1) || !in_offsets(at->v_token_stride, 0, 1))
        return GRKAN_ERR_UNSUPPORTED;
    if ((at->queries > 0 && at->batch > 0 && !at->q) || (at->keys > 0 && at->batch > 0 && (!at->k || !at->v)))
        return GRKAN_ERR_NULL;
    if (!fine_operand(at->q, at->q_batch_stride, at->q_token_stride, at->q_head_stride) ||
        !fine_operand(at->k, at->k_batch_stride, at->k_token_stride, at->k_head_stride) ||
        !fine_operand(at->v, at->v_batch_stride, at->v_token_stride, at->v_head_stride) ||
        reinterpret_cast<uintptr_t>(at->key_lengths) % (at->key_lengths_64 ? 8 : 4) != 0)
        return GRKAN_ERR_ALIGN;
    Args a = {};
    a.q = Operand{reinterpret_cast<uint64_t>(at->q), at->q_batch_stride * 2, at->q_token_stride * 2, at->q_head_stride * 2};
    a.k = Operand{reinterpret_cast<uint64_t>(at->k), at->k_batch_stride * 2, at->k_token_stride * 2, at->k_head_stride * 2};
    a.v = Operand{reinterpret_cast<uint64_t>(at->v), at->v_batch_stride * 2, at->v_token_stride * 2, at->v_head_stride * 2};
    a.lengths = at->key_lengths;
    a.lengths_64 = at->key_lengths_64;
    a.mask = static_cast<const uint8_t *>(at->key_mask);
    a.mask_batch = at->mask_batch_stride;
    a.mask_key = at->mask_key_stride;
    a.keys = at->keys;
    a.rows = at->queries * group;
    a.batch = (int32_t)at->batch;
    a.kv_heads = at->kv_heads;
    a.group = (int32_t)group;
    a.dim = at->dim;
    a.scale = at->scale;
    a.c = at->scale * 1.4426950408889634f;
    *to = a;
    return GRKAN_OK;
}

typedef void (*Kernel)(Args);
struct Variant {
    Kernel kernel, join;
    bool few; // rows
    int rows, keys, threads; // of a workgroup: rows, keys at a time
    size_t lds;
};

template <typename IO, int DP> static Variant pick(bool few)
{
    if (few)
        return Variant{tokens_kernel<TokenShape<IO, DP>>, join_tokens_kernel<IO>, true, 32, kGroup, 64 * TokenShape<IO, DP>::kWaves, TokenShape<IO, DP>::kLds};
    return Variant{forward_kernel<Shape<IO, DP>>, join_kernel<IO>, false, Shape<IO, DP>::kRows, Shape<IO, DP>::KT, 256, Shape<IO, DP>::kLds};
}
template <typename IO> static Variant pick(int32_t dim, bool few)
{
    return dim <= 32 ? pick<IO, 32>(few) : dim <= 64 ? pick<IO, 64>(few) : dim <= 96 ? pick<IO, 96>(few) : pick<IO, 128>(few);
}

// Whether the four wavefronts of a workgroup share the keys of 32 rows, instead of having 32 rows each.  Measured, in us (four times 32 rows / 32):
//   * where no compute unit, or with 64 channels only every other, has more than one workgroup, and the walk is neither over at once nor worth a split over several.  96 heads of 64 channels, one
//     row: 64 keys 5.2 / 5.8, 200 8.1 / 6.4, 400 10.4 / 8.8, 1,600 14 / 17; twelve with 128 rows: 577 keys 14.8 / 10.3, 1,500 13.9 / 18.2.
//     With 128 channels: 200 keys 10.4 / 10.2, 800 17 / 20; twelve with 128 rows: 577 keys 17.3 / 15.8.
//   * single tokens on long keys of uneven lengths, which are dealt out evenly.  300 heads, 5,000 keys at most, 64 channels 78 / 55, 128 channels 134 / 108; 768 heads
//     of 128 272 / 236; 96 heads 25 / 24 and 32 / 37.
static bool shares_keys(const Args &a, int64_t heads)
{
    const int64_t work = heads * ((a.rows + 31) / 32);
    if (a.keys > 128 && (a.dim <= 64 ? work <= kWorkers + kWorkers / 2 && a.keys <= 896 : work <= kWorkers && a.keys <= 640))
        return true;
    return a.rows <= 32 && a.lengths && a.keys > 2048 && heads >= 128;
}

// Over how many workgroups the keys of each of `base` are split, four tiles each at least: what takes the least time, counted in tiles of one
// that has a compute unit for itself.  Two there take 1.1 times as long as one, more as much longer as they are, up to `together`, and the
// others behind them; a split's beginning takes two tiles, the second launch six, or four of more than 64 channels, and the parts' way through
// memory, `rows` each, one for 6 MB, or 8 (`tile`: how much longer than in the forward pass a tile takes).  (us without and with: three batch entries with 700 queries, 5,000 keys, sixteen heads of 64, which are 288
// workgroups, 107 / 76; 300 heads of 128, one query, 5,000 keys 159 / 146.)
int64_t splits_of(int64_t base, int64_t tiles, int64_t rows, int64_t dim, double together, double tile)
{
    const double second = (dim <= 64 ? 6.0 : 4.0) / tile, bytes = (dim <= 64 ? 6e6 : 8e6) * tile;
    int64_t best = 1;
    double least = 0;
    auto look = [&](int64_t n) {
        if (n < 1 || (n > 1 && (base < 1 || 4 * n > tiles)))
            return;
        const double all = (double)base * (double)n, each = std::ceil(all / 256.0), rounds = std::floor(each / together), rest = each - rounds * together;
        const double share = rounds * 0.55 * together + (rest > 0 ? std::max(1.0, 0.55 * rest) : 0.0);
        const double cost = (double)((tiles + n - 1) / n + 2) * share + (n > 1 ? second + all * (double)(rows * dim) * 8.0 / bytes : 0.0);
        if (n == 1 || cost < least) {
            best = n;
            least = cost;
        }
    };
    for (int64_t n = 1; n <= 8; ++n)
        look(n);
    if (base > 0 && base < 64)
        for (int64_t most : {256, 512}) {
            const int64_t n = most / base;
            look(n < tiles / 4 ? n : tiles / 4);
        }
    return best;
}

// The kernel, and how the keys are split.
static Variant plan(Args &a, grkan_dtype_t io)
{
    const int64_t heads = (int64_t)a.batch * a.kv_heads;
    const bool few = shares_keys(a, heads);
    const Variant v = io == GRKAN_BF16 ? pick<__bf16>(a.dim, few) : pick<_Float16>(a.dim, few);
    const int64_t tiles = (a.keys + v.keys - 1) / v.keys;
    if (few) {
        a.row_tiles = (int32_t)((a.rows + 31) / 32);
        a.splits = 0;
        if (a.row_tiles > 1)
            return v;
        // A worker on every compute unit, with 256 keys at least; none where a key head each does as well: 1,024 of them, or all short
        // (the second launch takes as long as 1,024 keys one behind the other).
        const int64_t most = heads * tiles / 2;
        a.splits = heads >= 1024 || tiles <= 8 || most <= heads || heads * tiles >= (int64_t)1 << 30 ? 0 : (int32_t)(most < kWorkers ? most : kWorkers);
        return v;
    }
    a.row_tiles = (int32_t)((a.rows + v.rows - 1) / v.rows);
    const int64_t splits = splits_of(heads * a.row_tiles, tiles, a.rows < v.rows ? a.rows : v.rows, a.dim, a.dim <= 64 ? 4 : 2, 1.0);
    a.tiles_per_split = (int32_t)((tiles + splits - 1) / splits);
    if (a.tiles_per_split < 1)
        a.tiles_per_split = 1;
    a.splits = (int32_t)((tiles + a.tiles_per_split - 1) / a.tiles_per_split);
    if (a.splits < 1)
        a.splits = 1;
    return v;
}

// of the parts, where there are any
static size_t forward_bytes(const Args &a, const Variant &v)
{
    const size_t heads = (size_t)a.batch * (size_t)a.kv_heads;
    const size_t parts = v.few ? (a.splits > 0 ? heads + (size_t)a.splits : 0) : a.splits > 1 ? heads * (size_t)a.splits : 0;
    return parts * (size_t)a.rows * (size_t)(a.dim + 1) * sizeof(float);
}

size_t backward_bytes(const Args &a); // grkan_attention_bwd.hip

} // namespace attention
} // namespace grkan

using namespace grkan;

extern "C" size_t grkan_attention_lse_count(const grkan_attention_t *at)
{
    if (!at || at->batch < 0 || at->queries < 0 || at->heads < 0)
        return 0;
    return (size_t)at->batch * (size_t)at->queries * (size_t)at->heads;
}

extern "C" size_t grkan_attention_workspace_bytes(const grkan_attention_t *at, int32_t backward)
{
    attention::Args a;
    if (attention::fill(at, GRKAN_BF16, &a) != GRKAN_OK)
        return 0;
    if (backward)
        return attention::backward_bytes(a);
    return attention::forward_bytes(a, attention::plan(a, GRKAN_BF16));
}

extern "C" grkan_status_t grkan_attention_fwd(const grkan_attention_t *at, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                              grkan_dtype_t io, void *hip_stream)
{
    attention::Args a;
    const grkan_status_t bad = attention::fill(at, io, &a);
    if (bad != GRKAN_OK)
        return bad;
    if ((int64_t)a.batch * a.rows == 0)
        return GRKAN_OK;
    if (!out)
        return GRKAN_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(out) % 16 != 0 || reinterpret_cast<uintptr_t>(lse) % 4 != 0)
        return GRKAN_ERR_ALIGN;
    const attention::Variant v = attention::plan(a, io);
    const size_t need = attention::forward_bytes(a, v);
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
        return GRKAN_ERR_WORKSPACE;
    const int64_t heads = (int64_t)a.batch * a.kv_heads, work = v.few ? (a.splits > 0 ? a.splits : heads * a.row_tiles) : heads * a.row_tiles * a.splits;
    const int64_t join = !need ? 0 : v.few ? heads : (heads * a.rows * (a.dim / 8) + 255) / 256;
    if (work > attention::kMostBlocks || join > attention::kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    const int64_t grid = v.few ? work : attention::spread(a, work, (int64_t)a.row_tiles * a.splits);
    if (grid > attention::kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    a.out = static_cast<char *>(out);
    a.lse = lse;
    a.partial = static_cast<float *>(workspace);
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    if (!attention::allow_lds(reinterpret_cast<const void *>(v.kernel), v.lds))
        return GRKAN_ERR_LAUNCH;
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3((unsigned)grid), dim3((unsigned)v.threads), args, v.lds, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    if (join > 0 && hipLaunchKernel(reinterpret_cast<const void *>(v.join), dim3((unsigned)join), dim3(256), args, 0, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    return GRKAN_OK;
}
