// A cache of keys and values in pages, on gfx950 (MI355X): new tokens' keys and values into it, and attention of the newest tokens over it.
//
// Position p of sequence s lies in row p mod page_size of page table[s][p / page_size].  Of the `queries` newest tokens of a sequence of `length`, token i sees
// the positions up to length - queries + i: out_i = sum_p softmax_p(scale q_i k_p) v_p.
//
// The keys and values are read once, which bounds it: there are few rows for each.  As cross attention's kernel for single tokens (grkan_attention.hip), from the same
// parts: the four wavefronts of a workgroup take tiles of 32 keys each, without a barrier, and join what they found; the keys of all sequences and heads are dealt
// out evenly, in groups of 128, to a workgroup on each compute unit, and a second launch joins the parts.  Where the pages are whole tiles a tile has one address;
// elsewhere every lane has its key's.  The table's entries come to LDS in front of the walk, so that no load waits for another one within it.
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
    int32_t unit_rows; // of a part: 32, or all where they are fewer
};

// Walks over a sequence's keys: each key head and tile of 32 rows.
__device__ __forceinline__ int32_t units_of(const Paged &a) { return a.kv_heads * a.row_tiles; }

constexpr int kWorkers = 256;
constexpr int kEntries = 2048; // of the table in LDS at once

template <typename IO_, int DP_> struct PagedShape : TokenShape<IO_, DP_> {
    using Base = TokenShape<IO_, DP_>;
    static constexpr uint32_t kTable = (uint32_t)Base::kLds;
    static constexpr size_t kLds = Base::kLds + kEntries * 4;
};

template <class SH> __global__ __launch_bounds__(256, SH::DP > 64 ? 1 : 2) void paged_kernel(const Paged a)
{
    constexpr int DP = SH::DP, KT = SH::KT;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    int32_t *const table = reinterpret_cast<int32_t *>(smem + SH::kTable);
    const bool shared = a.splits > 0;
    const int32_t worker = (int32_t)blockIdx.x;
    const bool even = a.page % KT == 0; // a tile is in one page

    const TileLoads<DP, KT, 1> k_loads(0, lane, a.k.token, a.dim), v_loads(0, lane, a.v.token, a.dim);

    // groups [g0, g1) of walk `unit` of a sequence
    auto part = [&](int32_t b, int32_t unit, int32_t count, int32_t g0, int32_t g1) {
        const int32_t row_tile = unit / a.kv_heads, kvh = unit - row_tile * a.kv_heads;
        const uint32_t row0 = 32u * (uint32_t)row_tile, row = row0 + col, group = (uint32_t)a.group;
        const uint32_t rows_end = row0 + 32u < (uint32_t)a.rows ? row0 + 32u : (uint32_t)a.rows;
        Rows<typename SH::IO, DP, KT> rows;
        rows.load(a, b, kvh, row, h);
        // of the rows the last keys: the lane's, the first row's, and the last row's, behind which there are no keys for the tile of rows
        const int32_t before = count - a.queries;
        const Later later{before + (int32_t)(row / group), before + (int32_t)(row0 / group)};
        const int32_t seen = before + (int32_t)((rows_end - 1) / group) + 1, end = g1 * kGroup < seen ? g1 * kGroup : seen;
        const int32_t chunk = (kEntries - 1) / kGroup * kGroup; // keys, with page >= 1
        const uint64_t k_head = a.k.at + (uint64_t)(kvh * a.k.head), v_head = a.v.at + (uint64_t)(kvh * a.v.head);
        bool each = false;
        for (;;) {
            rows.clear();
            bool some = false;
#pragma unroll 1
            for (int64_t key0 = (int64_t)g0 * kGroup; key0 < end; key0 += (int64_t)chunk * a.page) {
                const int64_t behind = key0 + (int64_t)chunk * a.page;
                const int32_t key1 = behind < end ? (int32_t)behind : end, first = (int32_t)key0 / a.page, last = (key1 - 1) / a.page;
                const int32_t *const from = a.table + (int64_t)b * a.table_stride;
                barrier(); // (all are done with the entries before)
                for (int32_t i = first + tid; i <= last; i += 256) {
                    const int32_t page = from[i];
                    table[i - first] = page >= 0 && page < a.pages ? page : -1;
                }
                wait_loads<0>();
                barrier();
                int32_t page = -1, place = 0; // even: of the tile; else of key t KT + lane mod 32
                some |= walk_alone<SH>(
                    rows, (int32_t)(key0 / KT) + wave, (key1 + KT - 1) / KT, lds0, wave, lane, a.c, a.dim,
                    [&](int32_t t) -> uint64_t {
                        const int32_t left = key1 - t * KT;
                        const uint64_t below = left >= KT ? rows.kAll : ((uint64_t)1 << left) - 1u;
                        if (even) {
                            const int32_t entry = t * KT / a.page;
                            page = __builtin_amdgcn_readfirstlane(table[entry - first]);
                            place = t * KT - entry * a.page;
                            return page >= 0 ? below : 0;
                        }
                        const int32_t key = t * KT + (int32_t)col, entry = key / a.page;
                        place = key - entry * a.page;
                        page = key < key1 ? table[entry - first] : -1;
                        return below & __ballot(page >= 0);
                    },
                    [&](int32_t t, uint64_t word, bool whole, uint32_t to) {
                        if (even) {
                            k_loads.issue(k_head + (uint64_t)(page < 0 ? 0 : page) * (uint64_t)a.k.batch + (uint64_t)place * (uint64_t)a.k.token, a.k.token, word, whole, to);
                            v_loads.issue(v_head + (uint64_t)(page < 0 ? 0 : page) * (uint64_t)a.v.batch + (uint64_t)place * (uint64_t)a.v.token, a.v.token, word, whole,
                                          to + SH::kTile);
                            return;
                        }
                        using Loads = TileLoads<DP, KT, 1>;
#pragma unroll 1
                        for (int turn = 0; turn < Loads::kTurns; ++turn)
#pragma unroll
                            for (int q = 0; q < Loads::kEach; ++q) {
                                const uint32_t e = (uint32_t)q * 64u + (uint32_t)lane, r0 = e / Loads::kChunks, piece = (e % Loads::kChunks) ^ swizzle<DP>(r0);
                                const int32_t r = (int32_t)(r0 + Loads::kTokens * (uint32_t)turn);
                                const int64_t p = __shfl(page, r), i = __shfl(place, r);
                                const bool there = p >= 0 && (word >> r & 1u) && piece * 8u < (uint32_t)a.dim;
                                const uint64_t zeros = reinterpret_cast<uint64_t>(kZeros);
                                const uint32_t at = to + (uint32_t)(turn * Loads::kEach + q) * kBlock<DP>;
                                load_to_lds_at(there ? k_head + (uint64_t)(p * a.k.batch + i * a.k.token) + piece * 16u : zeros, at);
                                load_to_lds_at(there ? v_head + (uint64_t)(p * a.v.batch + i * a.v.token) + piece * 16u : zeros, at + SH::kTile);
                            }
                    },
                    later, each);
            }
            if (!some) // (a query may hold NaN, and masked keys' scores are 0 NaN then)
                rows.clear();
            // (all wavefronts, for the barriers)
            if (each || __syncthreads_or(rows.not_finite()) == 0)
                break;
            each = true;
        }
        const int64_t unit_at = (int64_t)b * units_of(a) + unit, slot = unit_at + worker;
        char *const out = shared ? reinterpret_cast<char *>(a.partial + (slot * a.unit_rows + col) * a.dim) : out_row(a, b, kvh, row);
        float *const lse = a.partial + (shared ? ((int64_t)a.batch * units_of(a) + a.splits) * a.unit_rows * a.dim + slot * a.unit_rows + col : 0);
        join_wavefronts<SH>(rows, smem, wave, lane, (int64_t)row < a.rows, a, out, lse, shared);
    };

    if (!shared) {
        const int32_t units = units_of(a), b = worker / units, count = keys_of(a, b);
        part(b, worker - b * units, count, 0, DealOf<Paged>::groups_of(count));
        return;
    }
    DealOf<Paged> deal(a);
    if (worker >= deal.workers)
        return;
    int32_t x = deal.first_of(worker);
    const int32_t end = deal.first_of(worker + 1);
    deal.find(a, x);
    while (x < end) {
        const int32_t unit = (x - deal.begin) / deal.groups, g0 = x - deal.begin - unit * deal.groups;
        const int32_t g1 = end - x < deal.groups - g0 ? g0 + end - x : deal.groups;
        part(deal.b, unit, deal.count, g0, g1);
        x += g1 - g0;
        if (x < end && x == deal.begin + deal.groups * units_of(a)) { // the next sequence with keys
            deal.begin = x;
            do {
                deal.count = keys_of(a, ++deal.b);
                deal.groups = DealOf<Paged>::groups_of(deal.count);
            } while (deal.groups == 0);
        }
    }
}

// out of the workers' parts: a workgroup for each walk, dim / 8 lanes a row, or sixteen times as many at most where the rows leave lanes over
template <typename IO> __global__ __launch_bounds__(256) void join_paged_kernel(const Paged a)
{
    const int32_t units = units_of(a), b = (int32_t)blockIdx.x / units, unit = (int32_t)blockIdx.x - b * units;
    const int32_t row_tile = unit / a.kv_heads, kvh = unit - row_tile * a.kv_heads;
    DealOf<Paged> deal(a);
    deal.find(a, -1, b);
    const int32_t x0 = deal.begin + unit * deal.groups;
    const int32_t w0 = deal.groups ? deal.worker_of(x0) : 0, parts = deal.groups ? deal.worker_of(x0 + deal.groups - 1) - w0 + 1 : 0;
    const uint32_t pieces = (uint32_t)a.dim / 8u, row0 = 32u * (uint32_t)row_tile;
    const uint32_t rows = (uint32_t)a.rows - row0 < 32u ? (uint32_t)a.rows - row0 : 32u;
    const float *const stats = a.partial + ((int64_t)a.batch * units + a.splits) * a.unit_rows * a.dim;
    const uint32_t items = rows * pieces;
    uint32_t lanes = 1;
    while (lanes < 16 && items * lanes * 2 <= 256)
        lanes *= 2;
    const uint32_t sub = threadIdx.x & (lanes - 1);
    for (uint32_t i = threadIdx.x / lanes; i < items; i += 256 / lanes) {
        const uint32_t row = i / pieces, piece = i - row * pieces;
        auto line = [&](int32_t p) { return ((int64_t)blockIdx.x + w0 + p) * a.unit_rows + row; };
        join_parts<IO>(
            parts, (int32_t)sub, (int32_t)lanes, [&](int32_t p) { return a.partial + line(p) * a.dim + 8u * piece; }, [&](int32_t p) { return stats[line(p)]; },
            out_row(a, b, kvh, row0 + row) + 16u * piece);
    }
}

// ------------------------------------------------------------------------------------------------ into the pages

struct PagedWrite : Packed { // k, v: of the new tokens; rows: tokens
    char *k_pages, *v_pages;
    int64_t k_page, k_place, k_place_head, v_page, v_place, v_place_head; // bytes
    const int32_t *table;
    const void *lengths;
    int64_t table_stride, pages;
    int32_t lengths_64, page, entries;
    int32_t per; // tokens of a workgroup, 64 at most
};

// A copy, 16 bytes a lane: bound by memory, or for few tokens by the way from the offsets over the lengths and the table to the page.
__global__ __launch_bounds__(256) void paged_write_kernel(const PagedWrite a)
{
    __shared__ int32_t page_of[64], place_of[64];
    const int32_t token0 = (int32_t)blockIdx.x * a.per, here = a.tokens - token0 < a.per ? a.tokens - token0 : a.per;
    if (threadIdx.x < 64) {
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
    if (q->tokens >= most || rows >= most || (rows + 31) / 32 * c->kv_heads >= most)
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
    a.row_tiles = (int32_t)((rows + 31) / 32);
    a.unit_rows = rows < 32 ? (int32_t)rows : 32;
    // A worker on every compute unit, with 256 keys at least; none where a walk each does as well: 1,024 of them, or all short.
    const int64_t walks = (int64_t)a.batch * a.kv_heads * a.row_tiles, groups = (a.keys + kGroup - 1) / kGroup, parts = walks * groups / 2;
    a.splits = walks >= 1024 || groups <= 8 || parts <= walks || walks * groups >= most ? 0 : (int32_t)(parts < kWorkers ? parts : kWorkers);
    *to = a;
    return GRKAN_OK;
}

static size_t workspace_of(const Paged &a)
{
    return a.splits > 0 ? ((size_t)a.batch * (size_t)a.kv_heads * (size_t)a.row_tiles + (size_t)a.splits) * (size_t)a.unit_rows * (size_t)(a.dim + 1) * sizeof(float) : 0;
}

typedef void (*Kernel)(Paged);
struct PagedVariant {
    Kernel kernel, join;
    size_t lds;
};
template <typename IO, int DP> static PagedVariant variant()
{
    return PagedVariant{paged_kernel<PagedShape<IO, DP>>, join_paged_kernel<IO>, PagedShape<IO, DP>::kLds};
}
template <typename IO> static PagedVariant pick(int32_t dim)
{
    return dim <= 32 ? variant<IO, 32>() : dim <= 64 ? variant<IO, 64>() : dim <= 96 ? variant<IO, 96>() : variant<IO, 128>();
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
    const int64_t walks = (int64_t)a.batch * a.kv_heads * a.row_tiles, work = a.splits > 0 ? a.splits : walks;
    if (work > attention::kMostBlocks || (need && walks > attention::kMostBlocks))
        return GRKAN_ERR_UNSUPPORTED;
    a.out = static_cast<char *>(out);
    a.partial = static_cast<float *>(workspace);
    const attention::PagedVariant v = io == GRKAN_BF16 ? attention::pick<__bf16>(a.dim) : attention::pick<_Float16>(a.dim);
    if (!attention::allow_lds(reinterpret_cast<const void *>(v.kernel), v.lds))
        return GRKAN_ERR_LAUNCH;
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3((unsigned)work), dim3(256), args, v.lds, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    if (need && hipLaunchKernel(reinterpret_cast<const void *>(v.join), dim3((unsigned)walks), dim3(256), args, 0, stream) != hipSuccess)
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
    if (tokens >= (int64_t)1 << 30 || (int64_t)cache->kv_heads * cache->dim >= (int64_t)1 << 24 || cache->sequences >= 1 << 30)
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
    a.per = (int32_t)(per < 64 ? per : 64);
    const int64_t grid = (tokens + a.per - 1) / a.per;
    if (grid > attention::kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    attention::paged_write_kernel<<<dim3((unsigned)grid), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(a);
    return hipGetLastError() == hipSuccess ? GRKAN_OK : GRKAN_ERR_LAUNCH;
}
