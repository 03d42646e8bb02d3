// Causal attention over packed sequences on gfx950 (MI355X), forward: row r of a sequence (a token's query of one head) sees the sequence's
// keys up to its own token's,
//
//     out_r = sum_{j <= r} exp(scale q_r k_j - m_r) v_j / sum_{j <= r} exp(scale q_r k_j - m_r)
//
// in one pass with the running maximum and sum, as cross attention does it (grkan_attention.hip), from the same parts: the queries of the
// heads that share a key head are one list of rows, and the probabilities go from the products of the scores to those of the values in
// registers. Products and masks stop at the diagonal: a workgroup ends at its last row's key, a wavefront leaves out tiles behind its own,
// and only the tiles that the diagonal crosses take comparisons.  The longest walks are launched first.
//
// What bounds it: the products and the exponentials of long sequences, which overlap little, and the card's clock, which falls under them
// (4,096 tokens, 32 heads of 128 on eight, float16: 139 us, 0.99 PFLOP/s, where a product of 8,192 has 1.37); of short ones the longest
// walk, a tile after the other, behind 5 us of launch, search and first loads (24 sequences of 60 to 1,000 tokens, twelve heads of 64: 21
// us, and 19 where both products are left out).
//
// A later token has no influence on an earlier one, NaN and infinities included: in the tiles on the diagonal its weight is zero, but zero
// times NaN is NaN.  Rows whose sums are not finite at the end are gone through a second time with those tiles row by row (Rows::add_each).
//
// The output is rounded once.  For the backward pass what that took away is kept, rounded too (`rest`).
#include <hip/hip_runtime.h>

#include <cmath>

#include "grkan_attention_rows.h"
#include "grkan_packed.h"
#include "grkan_turns.h"

namespace grkan {
namespace attention {

// Zeros, and an lse that gives no probability, for 32 rows that belong to no sequence.
template <int DP> __device__ __forceinline__ void clear_rows(const Packed &a, const Segment &s, int32_t kvh, uint32_t row0, int32_t rows, int lane)
{
    const uint32_t row = row0 + ((uint32_t)lane & 31u), h = (uint32_t)lane >> 5;
    if ((int32_t)row >= rows)
        return;
    const int64_t at = packed_at(a, s, kvh, row);
    for (int32_t channel = 8 * (int32_t)h; channel < a.dim; channel += 16) {
        *reinterpret_cast<u32x4 *>(a.out + at + 2 * channel) = u32x4{};
        if (a.rest)
            *reinterpret_cast<u32x4 *>(a.rest + at + 2 * channel) = u32x4{};
    }
    if (h == 0 && a.lse)
        a.lse[(int64_t)kvh * a.rows + packed_row(a, s, row)] = __builtin_inff();
}

// ------------------------------------------------------------------------------------------------ 32 rows a wavefront, tiles of 64 keys for all

// Two wavefronts' sums of the same rows (`pairs` of them, this is number `own`): the second leaves its own in LDS (and is done: false), the
// first adds them, relative to a common maximum.
template <class R> __device__ __forceinline__ bool join_two(R &rows, char *smem, int pairs, int own, int second, int lane, float c)
{
    constexpr int ND = R::ND;
    f32x4 *const sums = reinterpret_cast<f32x4 *>(smem) + own * ND * 4 * 64 + lane;
    float *const stats = reinterpret_cast<float *>(smem + pairs * ND * 4 * 64 * 16) + own * 2 * 64 + lane;
    if (second) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[j] = rows.acc[d][4 * g + j];
                sums[(4 * d + g) * 64] = o;
            }
        stats[0] = rows.top;
        stats[64] = rows.sum;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    if (second)
        return false;
    const float other = stats[0], top = fmaxf(rows.top, other), low = top > -__builtin_inff() ? top : 0.0f;
    const float mine = __builtin_amdgcn_exp2f((rows.top - low) * c), its = __builtin_amdgcn_exp2f((other - low) * c);
    rows.top = top;
    rows.sum = rows.sum * mine + stats[64] * its;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 o = sums[(4 * d + g) * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                rows.acc[d][4 * g + j] = rows.acc[d][4 * g + j] * mine + o[j] * its;
        }
    return true;
}

// The lane's row: of the output, what its rounding left, and the row's lse.
template <class R> __device__ __forceinline__ void store_rows(const R &rows, const Packed &a, const Segment &s, int32_t kvh, uint32_t row, int32_t all, uint32_t h)
{
    using MM = typename R::MM;
    if ((int32_t)row >= all)
        return;
    const float sum = halves_sum(rows.sum), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t at = packed_at(a, s, kvh, row);
#pragma unroll
    for (int d = 0; d < R::ND; ++d)
        store_channels<typename R::Type>(rows.acc[d], d, inv, a, a.out + at, false, h);
    if (a.rest) {
#pragma unroll
        for (int d = 0; d < R::ND; ++d) {
            f32x16 left;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = rows.acc[d][i] * inv, y = rows.acc[d][i + 1] * inv;
                const uint32_t w = MM::two(x, y);
                left[i] = x - MM::first(w);
                left[i + 1] = y - MM::second(w);
            }
            store_channels<typename R::Type>(left, d, 1.0f, a, a.rest + at, false, h);
        }
    }
    if (h == 0 && a.lse)
        a.lse[(int64_t)kvh * a.rows + packed_row(a, s, row)] = lse_of(log2_sum(rows.top, sum, a.c));
}

// PARTS: wavefronts that share the keys of a tile, of 32 rows each; the others have rows of their own.
template <typename IO_, int DP_, int PARTS_> struct CausalShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, PARTS = PARTS_, KT = 64, kKeys = KT / PARTS, kWaves = 4, kRows = 32 * kWaves / PARTS;
    static constexpr uint32_t kTile = kTileBytes<DP, KT>;
    static constexpr uint32_t kFlag = 4 * kTile; // behind K and V, two of each
    static constexpr size_t kLds = kFlag + 16;
    static_assert(PARTS == 1 || (DP / 8 * 64 * 16 + 2 * 64 * 4) * (kWaves / 2) <= kFlag, ""); // what the wavefronts join
};

template <class SH> __global__ __launch_bounds__(256, SH::DP <= 64 ? 4 : 2) void causal_kernel(const Packed a)
{
    constexpr int DP = SH::DP, KT = SH::KT, KEYS = SH::kKeys, ND = DP / 32;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5, group = (uint32_t)a.group;
    const int rows_of = wave / SH::PARTS, part = wave % SH::PARTS;

    const int32_t turn = (int32_t)blockIdx.x / a.kv_heads, kvh = (int32_t)blockIdx.x - turn * a.kv_heads;
    const Segment s = segment_of<SH::kRows>(a, turn, a.group, true);
    const int32_t all = s.count * a.group; // rows of the segment
    const int64_t begin = (int64_t)s.tile * SH::kRows;
    if (begin >= all)
        return;
    const uint32_t row0 = (uint32_t)begin + (uint32_t)rows_of * 32u, row = row0 + col;
    if (s.none) {
        if (part == 0)
            clear_rows<DP>(a, s, kvh, row0, all, lane);
        return;
    }
    // keys: of the workgroup up to its last row's, of the wavefront all below `from`, none from `to` on
    const int32_t end = (int32_t)((uint32_t)begin + SH::kRows - 1 < (uint32_t)all ? (uint32_t)begin + SH::kRows - 1 : (uint32_t)all - 1) / a.group + 1;
    const int32_t from = (int32_t)(row0 / group) + 1, to = (int32_t)((row0 + 31u) / group) + 1;
    const int32_t tiles = (end + KT - 1) / KT;
    const LastTwiceLoads<DP, KT, SH::kWaves> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    const uint64_t k_base = a.k.at + (uint64_t)((int64_t)s.first * a.k.token + kvh * a.k.head);
    const uint64_t v_base = a.v.at + (uint64_t)((int64_t)s.first * a.v.token + kvh * a.v.head);
    auto issue = [&](int32_t t, uint32_t at) {
        k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, a.k.token, a.dim, end - t * KT, lds0 + at);
        v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, a.v.token, a.dim, end - t * KT, lds0 + at + 2 * SH::kTile);
    };
    if (a.dim < DP) {
#pragma unroll 1
        for (uint32_t at = 0; at < 2 * SH::kTile; at += SH::kTile) {
            k_loads.clear(lane, lds0 + at);
            v_loads.clear(lane, lds0 + at + 2 * SH::kTile);
        }
    }
    issue(0, 0);
    Rows<typename SH::IO, DP, KEYS> rows;
    const uint32_t query = row / group;
    rows.load(a.q.at + (uint64_t)((int64_t)s.first * a.q.token + (int64_t)kvh * a.group * a.q.head + row_offset(row, group, a.q.token, a.q.head)),
              (int32_t)row < all, a.dim, h);
    arrived(rows.q);
    const bool works = (int32_t)row0 < all; // (a wavefront without rows loads for the others)
    // (two loops: one with a condition in it would copy the sums)
    auto walk = [&](auto each) {
        rows.clear();
        RowOperand<DP> k_from(lane);
        ColumnOperand<DP> v_from(lane);
        k_from.move(lds0 + row_at<DP>((uint32_t)(KEYS * part)));
        v_from.move(lds0 + row_at<DP>((uint32_t)(KEYS * part)) + 2 * SH::kTile);
        uint32_t at = 0;
#pragma unroll 1
        for (int32_t t = 0;;) { // (there is a tile: with a way past the loop it would copy the sums in every turn)
            wait_loads<0>();
            barrier(); // all wavefronts' loads of this tile are there, and all are done with the tile before
            if (t + 1 < tiles)
                issue(t + 1, at ^ SH::kTile);
            at ^= SH::kTile;
            if (t > 0) { // (K and V are moved alike)
                k_from.move(at ? 0u - SH::kTile : SH::kTile);
                v_from.move(at ? 0u - SH::kTile : SH::kTile);
            }
            const int32_t key0 = t * KT + KEYS * part; // the wavefront's first
            if (works && key0 < to) {
                f32x16 x[KEYS / 32];
                rows.template scores_ahead<2>(k_from, x);
                const bool crossed = key0 + KEYS > from;
                if (crossed)
                    rows.cut(x, (int32_t)query - key0, h);
                uint32_t p[KEYS / 32][8];
                rows.probabilities(x, a.c, p);
                bool apart = false;
                if constexpr (decltype(each)::value)
                    apart = crossed;
                if (apart)
                    rows.add_each(p, v_from, (int32_t)query - key0, col, h);
                else
                    rows.add(p, v_from);
            }
            if (++t == tiles)
                break;
        }
    };
    walk(std::false_type{});
    // (by all wavefronts, which load for one another)
    uint32_t *const flag = reinterpret_cast<uint32_t *>(smem + SH::kFlag);
    if (lane == 0)
        flag[wave] = works && rows.not_finite();
    wait_loads<0>();
    barrier();
    const int some = __builtin_amdgcn_readfirstlane((int)(flag[0] | flag[1] | flag[2] | flag[3]));
    if (__builtin_expect_with_probability(some != 0, 0, 1.0)) { // (its loops are not what registers go to)
        issue(0, 0);
        walk(std::true_type{});
        wait_loads<0>(); // (what is joined lies where the tiles were: all have read them in front of the barrier)
        barrier();
    }
    if constexpr (SH::PARTS > 1)
        if (!join_two(rows, smem, SH::kWaves / 2, rows_of, part, lane, a.c))
            return;
    store_rows(rows, a, s, kvh, row, all, h);
}

// The same with 256 rows and eight wavefronts, for heads of 128 channels, where the device holds two wavefronts of a SIMD: two groups of
// four take turns.  While the matrix units compute the products of one (the scores of a tile, and the values of the tile before: 1,160
// cycles), the vector unit has the probabilities of the other (1,000).  A barrier ends each turn; the second group is a turn behind, on the
// same tiles, which are loaded once for both, into the third place behind the two that are read from. Left to themselves the wavefronts of
// two workgroups come to do the same at the same time: 4,500 cycles for a tile of each, here 3,500, and a clock that falls from 1.95 to
// 1.88 GHz.
template <typename IO_, int DP_> struct TurnsShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, KT = 64, kRows = 256, kThreads = 512;
    static constexpr uint32_t kTile = kTileBytes<DP, KT>;
    static constexpr uint32_t kFlag = 6 * kTile; // behind K and V, three of each
    static constexpr size_t kLds = kFlag + 32;
};

template <class SH> __global__ __launch_bounds__(512, 2) void causal_turns_kernel(const Packed a)
{
    constexpr int DP = SH::DP, KT = SH::KT;
    extern __shared__ __align__(256) char smem[];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool second = wave >= 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5, group = (uint32_t)a.group;

    const int32_t turn = (int32_t)blockIdx.x / a.kv_heads, kvh = (int32_t)blockIdx.x - turn * a.kv_heads;
    const Segment s = segment_of<SH::kRows>(a, turn, a.group, true);
    const int32_t all = s.count * a.group; // rows of the segment
    const int64_t begin = (int64_t)s.tile * SH::kRows;
    if (begin >= all)
        return;
    const uint32_t row0 = (uint32_t)begin + (uint32_t)wave * 32u, row = row0 + col;
    if (s.none) {
        clear_rows<DP>(a, s, kvh, row0, all, lane);
        return;
    }
    // keys: of the workgroup up to its last row's, of the wavefront all below `from`
    const int32_t end = (int32_t)((uint32_t)begin + SH::kRows - 1 < (uint32_t)all ? (uint32_t)begin + SH::kRows - 1 : (uint32_t)all - 1) / a.group + 1;
    const int32_t from = (int32_t)(row0 / group) + 1, tiles = (end + KT - 1) / KT;
    const LastTwiceLoads<DP, KT, 8> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    const uint64_t k_base = a.k.at + (uint64_t)((int64_t)s.first * a.k.token + kvh * a.k.head);
    const uint64_t v_base = a.v.at + (uint64_t)((int64_t)s.first * a.v.token + kvh * a.v.head);
    // tile t, to its place
    auto load_keys = [&](int32_t t, uint32_t at) {
        if (t < tiles)
            k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, a.k.token, a.dim, end - t * KT, lds0 + at);
    };
    auto load_values = [&](int32_t t, uint32_t at) {
        if (t < tiles)
            v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, a.v.token, a.dim, end - t * KT, lds0 + at + 3 * SH::kTile);
    };
    load_keys(0, 0);
    Rows<typename SH::IO, DP, KT> rows;
    const uint32_t query = row / group;
    rows.load(a.q.at + (uint64_t)((int64_t)s.first * a.q.token + (int64_t)kvh * a.group * a.q.head + row_offset(row, group, a.q.token, a.q.head)),
              (int32_t)row < all, a.dim, h);
    arrived(rows.q);
    auto walk = [&](auto each) {
        rows.clear();
        RowOperand<DP> k_from(lane);
        ColumnOperand<DP> v_from(lane);
        k_from.move(lds0);
        v_from.move(lds0 + 3 * SH::kTile);
        f32x16 x[KT / 32];
        uint32_t p[KT / 32][8];
        auto wait = [&] { wait_loads<0>(); };
        auto meet = [&] {
            fence_schedule();
            barrier();
        };
        auto scores = [&] { rows.template scores_ahead<2>(k_from, x); };
        // (without conditions that would copy the sums: a wavefront's last tiles may be cut off as a whole)
        auto probabilities = [&](int32_t t, uint32_t at, uint32_t next) {
            const int32_t key0 = t * KT;
            if (key0 + KT > from)
                rows.cut(x, (int32_t)query - key0, h);
            rows.probabilities(x, a.c, p);
            // (here, and not where they are used first, in the other group's time)
#pragma unroll
            for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    asm volatile("" : "+v"(p[kb][j]));
            asm volatile("" : "+v"(rows.sum));
            k_from.move(next - at);
        };
        // (a load between eight products, as one waits for 100 cycles behind the others')
        auto products = [&](int32_t t, uint32_t at, uint32_t next, uint32_t last) {
            const int32_t key0 = t * KT;
            const bool spread = end - (t + 3) * KT >= KT && !decltype(each)::value;
            const uint64_t keys = uniform_u64(k_base + (uint64_t)(t + 3) * KT * (uint64_t)a.k.token);
            const uint64_t values = uniform_u64(v_base + (uint64_t)(t + 2) * KT * (uint64_t)a.v.token);
            if (!spread) {
                load_keys(t + 3, at);
                load_values(t + 2, last);
            }
            bool apart = false;
            if constexpr (decltype(each)::value)
                apart = key0 + KT > from;
            if (apart) {
                rows.scores(k_from, x);
                rows.add_each(p, v_from, (int32_t)query - key0, col, h);
            } else {
                rows.scores_and_add(k_from, x, p, v_from, [&](int n) {
                    if (spread) {
                        if (n < 2)
                            k_loads.one(n, keys, lds0 + at);
                        else
                            v_loads.one(n - 2, values, lds0 + last + 3 * SH::kTile);
                    }
                });
            }
            v_from.move(next - at);
        };
        take_turns<SH::kTile>(tiles, second, wait, meet, load_keys, load_values, scores, probabilities, products);
    };
    walk(std::false_type{});
    // (by all wavefronts, which load for one another)
    uint32_t *const flag = reinterpret_cast<uint32_t *>(smem + SH::kFlag);
    if (lane == 0)
        flag[wave] = (int32_t)row0 < all && rows.not_finite();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    uint32_t some = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w)
        some |= flag[w];
    if (__builtin_expect_with_probability(__builtin_amdgcn_readfirstlane((int)some) != 0, 0, 1.0)) {
        load_keys(0, 0);
        walk(std::true_type{});
    }
    store_rows(rows, a, s, kvh, row, all, h);
}

// ------------------------------------------------------------------------------------------------ host

static bool fine_operand(const void *p, int64_t token, int64_t head) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (token | head) % 8 == 0; }

grkan_status_t fill(const grkan_causal_attention_t *at, grkan_dtype_t io, Packed *to)
{
    if (!at)
        return GRKAN_ERR_NULL;
    if (at->tokens < 0 || at->sequences < 0 || at->heads < 1 || at->kv_heads < 1 || at->heads % at->kv_heads != 0 || at->dim < 1)
        return GRKAN_ERR_SHAPE;
    if (!at->offsets && (at->sequences == 0 ? at->tokens != 0 : at->tokens % at->sequences != 0))
        return GRKAN_ERR_SHAPE;
    if (io != GRKAN_BF16 && io != GRKAN_F16)
        return GRKAN_ERR_DTYPE;
    const int64_t group = at->heads / at->kv_heads;
    if (at->dim % 8 != 0 || at->dim > 128 || !(at->scale > 0) || !std::isfinite(at->scale * 1.4426950408889634f))
        return GRKAN_ERR_UNSUPPORTED;
    // rows, and tiles with them, are counted in 31 bits; offsets in a tile of 64 tokens too
    const int64_t most = (int64_t)1 << 30;
    if (group >= 1 << 20 || at->tokens >= most || at->tokens * group >= most || at->sequences >= most)
        return GRKAN_ERR_UNSUPPORTED;
    // every launch below 2^32 threads: tiles are of 64 rows or keys at least
    if ((at->tokens * group / 32 + at->sequences + 2) * at->kv_heads > kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    if (!in_offsets(at->q_token_stride, at->q_head_stride, group) || !in_offsets(at->k_token_stride, 0, 1) || !in_offsets(at->v_token_stride, 0, 1))
        return GRKAN_ERR_UNSUPPORTED;
    if (at->tokens > 0 && (!at->q || !at->k || !at->v))
        return GRKAN_ERR_NULL;
    if (!fine_operand(at->q, at->q_token_stride, at->q_head_stride) || !fine_operand(at->k, at->k_token_stride, at->k_head_stride) ||
        !fine_operand(at->v, at->v_token_stride, at->v_head_stride) || reinterpret_cast<uintptr_t>(at->offsets) % (at->offsets_64 ? 8 : 4) != 0)
        return GRKAN_ERR_ALIGN;
    Packed a = {};
    a.q = Operand{reinterpret_cast<uint64_t>(at->q), 0, at->q_token_stride * 2, at->q_head_stride * 2};
    a.k = Operand{reinterpret_cast<uint64_t>(at->k), 0, at->k_token_stride * 2, at->k_head_stride * 2};
    a.v = Operand{reinterpret_cast<uint64_t>(at->v), 0, at->v_token_stride * 2, at->v_head_stride * 2};
    a.rows = at->tokens * group;
    a.keys = at->tokens;
    a.batch = 1;
    a.kv_heads = at->kv_heads;
    a.group = (int32_t)group;
    a.dim = at->dim;
    a.scale = at->scale;
    a.c = at->scale * 1.4426950408889634f;
    a.offsets = at->offsets;
    a.offsets_64 = at->offsets_64;
    a.sequences = at->sequences;
    a.tokens = (int32_t)at->tokens;
    a.each = at->sequences > 0 ? (int32_t)(at->tokens / at->sequences) : 0;
    *to = a;
    return GRKAN_OK;
}

typedef void (*Kernel)(Packed);
struct CausalVariant {
    Kernel kernel;
    size_t lds;
    int64_t slots;
    int threads;
};
template <class SH> static CausalVariant four(const Packed &a)
{
    return CausalVariant{causal_kernel<SH>, SH::kLds, slots_of<SH::kRows>(a, a.group), 256};
}
template <class SH> static CausalVariant turns(const Packed &a)
{
    return CausalVariant{causal_turns_kernel<SH>, SH::kLds, slots_of<SH::kRows>(a, a.group), SH::kThreads};
}
template <typename IO, int DP> static CausalVariant pick(const Packed &a)
{
    return few_rows(a) ? four<CausalShape<IO, DP, 2>>(a) : four<CausalShape<IO, DP, 1>>(a);
}
template <typename IO> static CausalVariant pick(const Packed &a)
{
    // (turns: longer walks and fewer of them.  us without and with, query heads / key heads: one of 16,384 tokens, 8/2 537 / 466, of 4,096,
    // 32/32 148 / 139, 32/8 145 / 133, of 3,000, 32/8 83.2 / 81.8, four of 500 to 2,000, 32/8 59.7 / 56.2; too few workgroups: one of
    // 8,192, 8/8 165 / 175, of 2,048, 32/8 49 / 54; too short: four of 800 to 3,000, 16/16 61 / 69, eight of 60 to 1,000, 32/8 32 / 35.  The
    // host knows the average alone: long sequences beside many empty ones go without)
    if (a.dim == 128 && a.sequences > 0 && a.rows / a.sequences >= 4096 && slots_of<256>(a, a.group) * a.kv_heads >= 384)
        return turns<TurnsShape<IO, 128>>(a);
    return a.dim <= 32 ? pick<IO, 32>(a) : a.dim <= 64 ? pick<IO, 64>(a) : a.dim <= 96 ? pick<IO, 96>(a) : pick<IO, 128>(a);
}

// Two wavefronts on the tiles of 64 keys of the same rows where tiles of 128 rows do not fill the device (four workgroups of a compute unit, with
// more than 64 channels two): the longest walk is then what counts, and it is half as long.  us with 128 rows to a workgroup and with 64: twelve heads
// of 64 channels, 24 sequences of 60 to 1,000 tokens 21.1 / 19.9, eight of 120 to 2,000 31.5 / 25.1, one of 4,096 57 / 44, 30 of 60 to 1,000
// 22.4 / 23.6, 60 of 12 to 200 10.9 / 13.1, 16 of 240 to 4,000 110 / 136; 32 heads of 128 on eight, one of 1,500 36.0 / 34.9, of 2,000 46.9 / 51.4, eight of 60
// to 1,000 31.8 / 41.3; 16 of 96, 14 of 60 to 1,000 27.7 / 25.0, one of 6,000 131 / 143, 18 of 60 to 1,000 29.4 / 35.3.
bool few_rows(const Packed &a)
{
    return slots_of<128>(a, a.group) * a.kv_heads <= (a.dim <= 64 ? 1024 : a.dim <= 96 ? 720 : 448);
}

} // namespace attention
} // namespace grkan

using namespace grkan;

extern "C" size_t grkan_causal_attention_lse_count(const grkan_causal_attention_t *at)
{
    return !at || at->tokens < 0 || at->heads < 0 ? 0 : (size_t)at->tokens * (size_t)at->heads;
}

extern "C" grkan_status_t grkan_causal_attention_fwd(const grkan_causal_attention_t *at, void *out, void *rest, float *lse, grkan_dtype_t io,
                                                     void *hip_stream)
{
    attention::Packed a;
    const grkan_status_t bad = attention::fill(at, io, &a);
    if (bad != GRKAN_OK)
        return bad;
    if (a.tokens == 0)
        return GRKAN_OK;
    if (!out)
        return GRKAN_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(rest)) % 16 != 0 || reinterpret_cast<uintptr_t>(lse) % 4 != 0)
        return GRKAN_ERR_ALIGN;
    const attention::CausalVariant v = io == GRKAN_BF16 ? attention::pick<__bf16>(a) : attention::pick<_Float16>(a);
    const int64_t grid = v.slots * a.kv_heads;
    a.slots = (int32_t)v.slots;
    a.out = static_cast<char *>(out);
    a.rest = static_cast<char *>(rest);
    a.lse = lse;
    if (!attention::allow_lds(reinterpret_cast<const void *>(v.kernel), v.lds))
        return GRKAN_ERR_LAUNCH;
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3((unsigned)grid), dim3((unsigned)v.threads), args, v.lds,
                        static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    return GRKAN_OK;
}
