// Cross attention on gfx950 (MI355X), forward: out = softmax(scale Q K^T) V in one pass over the keys, with the running maximum and sum
// of each row.
//
//   * With rows enough (queries x heads that share a key head), a workgroup of four wavefronts has 32 each; 64 keys and their
//     values at a time come to LDS by LDS-direct loads, two tiles deep, and serve all four.
//   * With 32 rows or fewer (single tokens) the keys are what there is to read: the four wavefronts have the same rows and
//     tiles of 32 keys of their own, in LDS of their own, without a barrier, and join what they found at the end.
//   * Where the workgroups would not fill the chip, the keys are split over several, and a second launch joins them.
//
// The maximum of a row is raised only where a score passes it by more than 2^8 in the exponent: the probabilities are then at most 256,
// which neither 16-bit type minds, and the accumulators are scaled in few of the tiles instead of in most.
#include <hip/hip_runtime.h>

#include <cmath>
#include <mutex>
#include <unordered_set>

#include "grkan_attention.h"

namespace grkan {
namespace attention {

template <typename IO_, int DP_, bool KEYS_> struct Shape {
    typedef IO_ IO;
    static constexpr int DP = DP_, kWaves = 4;
    static constexpr bool KEYS = KEYS_;       // the wavefronts split the keys, not the rows
    static constexpr int KT = KEYS ? 32 : 64; // keys of a tile
    static constexpr int kRows = KEYS ? 32 : 32 * kWaves;
    static constexpr uint32_t kTile = kTileBytes<DP, KT>, kStage = 2 * kTile;
    static constexpr size_t kLds = (size_t)kStage * 2 * (KEYS ? kWaves : 1);
};

template <class SH> __global__ __launch_bounds__(256, 2) void forward_kernel(const Args a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, KT = SH::KT, KB = KT / 32, ND = DP / 32, NS = DP / 16;
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
    // ---- this wavefront's rows as second operands: lane l has row l mod 32, channels 16 s + 8 (l / 32) ..
    const uint32_t row0 = (uint32_t)row_tile * SH::kRows + (SH::KEYS ? 0u : (uint32_t)wave * 32u), row = row0 + col;
    u32x4 q[NS];
    {
        const uint64_t at = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head +
                                                row_offset(row, (uint32_t)a.group, a.q.token, a.q.head));
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool there = (int64_t)row < a.rows && channel < (uint32_t)a.dim;
            q[s] = gload16(there ? at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
    }

    const int32_t count = keys_of(a, b), tiles = (count + KT - 1) / KT;
    int32_t t0 = split * a.tiles_per_split, t1 = t0 + a.tiles_per_split;
    t1 = t1 < tiles ? t1 : tiles;
    if (SH::KEYS)
        t0 += wave;

    constexpr int loaders = SH::KEYS ? 1 : SH::kWaves;
    const TileLoads<DP, KT, loaders> k_loads(SH::KEYS ? 0 : wave, lane, a.k.token, a.dim), v_loads(SH::KEYS ? 0 : wave, lane, a.v.token, a.dim);
    const RowOperand<DP> k_operand(lane);
    const ColumnOperand<DP> v_operand(lane);
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
    ValidKeys valid(a, b, count);
    constexpr uint64_t all = KT == 64 ? ~(uint64_t)0 : 0xffffffffu;

    auto word_of = [&](int32_t t) {
        if constexpr (KT == 64)
            return valid.word(t);
        else
            return (valid.word(t / 2) >> (t % 2 * 32)) & all;
    };
    auto issue_k = [&](int32_t t, uint64_t word, uint32_t to) {
        k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, word, word == all && a.dim == DP, to);
    };
    auto issue_v = [&](int32_t t, uint64_t word, uint32_t to) {
        v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, word, word == all && a.dim == DP, to);
    };

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        acc[d] = f32x16{};
    float top = -__builtin_inff(), sum = 0.0f; // the maximum that the probabilities are relative to; this lane's part of their sum
    const float c = a.c, slack = fminf(8.0f / c, 1e38f); // (of scores)

    auto compute = [&](uint32_t k_at, uint32_t v_at, uint64_t word) {
        const auto k_from = k_operand.moved(k_at);
        const auto v_from = v_operand.moved(v_at);
        f32x16 s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            s[kb] = f32x16{};
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const u32x4 k = RowOperand<DP>::read(k_from, kb, st);
                s[kb] = MM::multiply(k, q[st], s[kb]);
            }
        if (word != all) { // keys that are not valid: minus infinity
            const uint64_t mine = word >> (4u * h);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const uint32_t bits = (uint32_t)(mine >> (32 * kb));
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[kb][i] = (bits >> (8 * (i / 4) + i % 4)) & 1u ? s[kb][i] : -__builtin_inff();
            }
        }
        uint32_t p[KB][8];
        float most = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                most = fmaxf(most, s[kb][i]);
        most = halves_max(most);
        if (__ballot(most > top + slack) != 0) {
            const float next = fmaxf(top, most);
            const float by = next > -__builtin_inff() ? __builtin_amdgcn_exp2f((top - next) * c) : 1.0f;
            top = next;
            sum *= by;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[d][i] *= by;
        }
        const float less = top > -__builtin_inff() ? top * c : 0.0f;
        float part = 0.0f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -less)), y = __builtin_amdgcn_exp2f(fmaf(s[kb][i + 1], c, -less));
                part += x + y;
                p[kb][i / 2] = MM::two(x, y);
            }
        sum += part;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const u32x4 v = ColumnOperand<DP>::read(v_from, kb, t, d);
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = p[kb][4 * t + j];
                    acc[d] = MM::multiply(v, w, acc[d]);
                }
    };

    if constexpr (SH::KEYS) {
        // tiles t0, t0 + 4, .. of this wavefront's own: loads of the next in flight while one is computed
        constexpr int kAhead = 2 * TileLoads<DP, KT, 1>::kMine;
        const uint32_t stages = lds0 + (uint32_t)wave * 2u * SH::kStage;
        uint32_t at = 0;
        uint64_t word = 0;
        if (t0 < t1) {
            word = word_of(t0);
            issue_k(t0, word, stages);
            issue_v(t0, word, stages + SH::kTile);
        }
        arrived(q);
        for (int32_t t = t0; t < t1; t += SH::kWaves) {
            uint64_t next = 0;
            if (t + SH::kWaves < t1) {
                next = word_of(t + SH::kWaves);
                issue_k(t + SH::kWaves, next, stages + (at ^ SH::kStage));
                issue_v(t + SH::kWaves, next, stages + (at ^ SH::kStage) + SH::kTile);
                wait_loads<kAhead>();
            } else {
                wait_loads<0>();
            }
            compute(stages + at, stages + at + SH::kTile, word);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (the tile's buffer is loaded into next)
            at ^= SH::kStage;
            word = next;
        }
    } else {
        const uint32_t ks = lds0, vs = lds0 + 2 * SH::kTile;
        const bool works = (int64_t)row0 < a.rows; // (a wavefront without rows loads for the others)
        uint32_t at = 0;
        uint64_t word = 0;
        if (t0 < t1) {
            word = word_of(t0);
            issue_k(t0, word, ks);
            issue_v(t0, word, vs);
        }
        arrived(q);
        for (int32_t t = t0; t < t1; ++t) {
            const uint64_t next = t + 1 < t1 ? word_of(t + 1) : 0;
            wait_loads<0>();
            barrier();
            if (t + 1 < t1) {
                issue_k(t + 1, next, ks + (at ^ SH::kTile));
                issue_v(t + 1, next, vs + (at ^ SH::kTile));
            }
            if (works)
                compute(ks + at, vs + at, word);
            at ^= SH::kTile;
            word = next;
        }
    }
    sum = halves_sum(sum);

    if constexpr (SH::KEYS) {
        // the four wavefronts' parts of each row: sums relative to a common maximum, added in wavefront order
        float *const joined = reinterpret_cast<float *>(smem); // [wave][channel][32 rows]
        float *const stats = joined + SH::kWaves * DP * 32;    // [wave][2][32 rows]
        wait_loads<0>();
        barrier();
        if (h == 0) {
            stats[wave * 64 + col] = top;
            stats[wave * 64 + 32 + col] = sum;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
        float most = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < SH::kWaves; ++w)
            most = fmaxf(most, stats[w * 64 + col]);
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < SH::kWaves; ++w) {
            const float m = stats[w * 64 + col];
            total += m > -__builtin_inff() ? stats[w * 64 + 32 + col] * __builtin_amdgcn_exp2f((m - most) * c) : 0.0f;
        }
        const float by = top > -__builtin_inff() ? __builtin_amdgcn_exp2f((top - most) * c) : 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                joined[(wave * DP + 32 * d + 8 * (i / 4) + 4 * (int)h + i % 4) * 32 + (int)col] = acc[d][i] * by;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
        top = most;
        sum = total;
        if (wave >= ND)
            return; // wavefront w writes channels 32 w ..
#pragma unroll
        for (int d = 0; d < ND; ++d)
            if (d == wave) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float *const from = joined + (32 * d + 8 * (i / 4) + 4 * (int)h + i % 4) * 32 + (int)col;
                    acc[d][i] = ((from[0] + from[DP * 32]) + from[2 * DP * 32]) + from[3 * DP * 32];
                }
            }
    }
    // ---- out: lane l has channels 32 d + 8 (i / 4) + 4 (l / 32) .. of row l mod 32
    const bool split_up = a.splits > 1;
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    char *const out0 = a.out + 2 * ((int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim);
    if ((int64_t)row >= a.rows)
        return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const float l2 = sum == 0.0f ? -__builtin_inff() : top * c + __builtin_amdgcn_logf(sum);
    const int64_t line = ((int64_t)split * a.batch * a.kv_heads + bh) * a.rows + row;
    char *const out = split_up ? reinterpret_cast<char *>(a.partial + line * a.dim)
                               : out0 + 2 * row_offset(row, (uint32_t)a.group, heads_dim, a.dim);
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        if (SH::KEYS && d != wave)
            continue;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int channel = 32 * d + 8 * g + 4 * (int)h;
            if (channel >= a.dim)
                continue;
            f32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[j] = acc[d][4 * g + j] * inv;
            if (split_up) {
                *reinterpret_cast<f32x4 *>(out + channel * 4) = o;
            } else {
                u32x2 w;
                w[0] = MM::two(o[0], o[1]);
                w[1] = MM::two(o[2], o[3]);
                *reinterpret_cast<u32x2 *>(out + channel * 2) = w;
            }
        }
    }
    if (h == 0 && (!SH::KEYS || wave == 0)) {
        if (split_up)
            a.partial[(int64_t)a.splits * a.batch * a.kv_heads * a.rows * a.dim + line] = l2;
        else if (a.lse)
            a.lse[line] = sum == 0.0f ? __builtin_inff() : l2;
    }
}

// out of the splits' rows, each the mean over its own keys, by the share of the sum that each has: dim / 8 lanes a row, eight channels each
template <typename IO> __global__ __launch_bounds__(256) void join_kernel(const Args a)
{
    const int64_t all = (int64_t)a.batch * a.kv_heads * a.rows;
    const uint32_t pieces = (uint32_t)a.dim / 8u;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, line = i / pieces;
    const uint32_t piece = (uint32_t)(i - line * pieces);
    if (line >= all)
        return;
    const float *const stats = a.partial + (int64_t)a.splits * all * a.dim;
    float most = -__builtin_inff();
    for (int32_t s = 0; s < a.splits; ++s)
        most = fmaxf(most, stats[s * all + line]);
    float total = 0.0f, o[8] = {};
    for (int32_t s = 0; s < a.splits; ++s) {
        const float l2 = stats[s * all + line];
        if (l2 == -__builtin_inff())
            continue; // no valid key in this split
        const float share = __builtin_amdgcn_exp2f(l2 - most);
        total += share;
        const f32x4 *const from = reinterpret_cast<const f32x4 *>(a.partial + (s * all + line) * a.dim + 8u * piece);
        const f32x4 x = from[0], y = from[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            o[j] += share * x[j];
            o[4 + j] += share * y[j];
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int64_t bh = line / a.rows;
    const uint32_t row = (uint32_t)(line - bh * a.rows);
    const int32_t b = (int32_t)(bh / a.kv_heads), kvh = (int32_t)(bh - (int64_t)b * a.kv_heads);
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    const int64_t first = (int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim;
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = Matrix<IO>::two(o[2 * j] * inv, o[2 * j + 1] * inv);
    *reinterpret_cast<u32x4 *>(a.out + (first + row_offset(row, (uint32_t)a.group, heads_dim, a.dim)) * 2 + 16u * piece) = w;
    if (a.lse && piece == 0)
        a.lse[line] = total == 0.0f ? __builtin_inff() : most + __builtin_amdgcn_logf(total);
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
    std::lock_guard<std::mutex> lock(mu);
    if (done[dev].count(kernel))
        return true;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
        return false;
    done[dev].insert(kernel);
    return true;
}

unsigned spread(Args &a, int64_t work, int64_t per_head)
{
    int64_t run = work / 64 < per_head ? work / 64 : per_head;
    run = run > 1 ? run : 1;
    a.work = (int32_t)work;
    a.run = (int32_t)run;
    return (unsigned)((work + 8 * run - 1) / (8 * run) * 8 * run);
}

static bool fine_operand(const void *p, int64_t batch, int64_t token, int64_t head)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (batch | token | head) % 8 == 0;
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
    if (at->dim % 8 != 0 || at->dim > 128 || !(at->scale > 0) || !std::isfinite(at->scale))
        return GRKAN_ERR_UNSUPPORTED;
    // rows and tiles are counted in 31 bits, offsets in a tile of 64 tokens too
    const int64_t most = (int64_t)1 << 31;
    if (at->batch >= most || at->keys > most - 256 || at->queries >= most || at->queries * group >= most - 256 || at->batch * at->kv_heads >= most)
        return GRKAN_ERR_UNSUPPORTED;
    for (const int64_t stride : {at->q_token_stride, at->k_token_stride, at->v_token_stride})
        if (stride < 0 || stride > (most - 512) / 128)
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
    Kernel kernel;
    int rows, keys; // of a workgroup, of a tile
    bool splits_keys;
    size_t lds;
};
template <class SH> static Variant variant() { return Variant{forward_kernel<SH>, SH::kRows, SH::KT, SH::KEYS, SH::kLds}; }

template <typename IO, int DP> static Variant pick(int64_t rows)
{
    if (rows <= 32)
        return variant<Shape<IO, DP, true>>();
    return variant<Shape<IO, DP, false>>();
}
template <typename IO> static Variant pick(int32_t dim, int64_t rows)
{
    return dim <= 32 ? pick<IO, 32>(rows) : dim <= 64 ? pick<IO, 64>(rows) : dim <= 96 ? pick<IO, 96>(rows) : pick<IO, 128>(rows);
}

// The kernel, its grid and how the keys are split.
static Variant plan(Args &a, grkan_dtype_t io)
{
    const Variant v = io == GRKAN_BF16 ? pick<__bf16>(a.dim, a.rows) : pick<_Float16>(a.dim, a.rows);
    a.row_tiles = (int32_t)((a.rows + v.rows - 1) / v.rows);
    const int64_t base = (int64_t)a.batch * a.kv_heads * a.row_tiles, tiles = (a.keys + v.keys - 1) / v.keys;
    // as many as give each compute unit two workgroups, each with four tiles for a wavefront at least
    const int64_t most = tiles / (v.splits_keys ? 16 : 4);
    int64_t splits = base > 0 && base < 384 ? 512 / base : 1;
    splits = splits < most ? splits : most;
    splits = splits > 1 ? splits : 1;
    a.tiles_per_split = (int32_t)((tiles + splits - 1) / splits);
    if (a.tiles_per_split < 1)
        a.tiles_per_split = 1;
    a.splits = (int32_t)((tiles + a.tiles_per_split - 1) / a.tiles_per_split);
    if (a.splits < 1)
        a.splits = 1;
    return v;
}

static size_t forward_bytes(const Args &a)
{
    return a.splits > 1 ? (size_t)a.splits * (size_t)a.batch * (size_t)a.kv_heads * (size_t)a.rows * (size_t)(a.dim + 1) * sizeof(float) : 0;
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
    attention::plan(a, GRKAN_BF16);
    return attention::forward_bytes(a);
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
    const size_t need = attention::forward_bytes(a);
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
        return GRKAN_ERR_WORKSPACE;
    const int64_t work = (int64_t)a.batch * a.kv_heads * a.row_tiles * a.splits;
    if (work > INT32_MAX / 2)
        return GRKAN_ERR_UNSUPPORTED;
    a.out = static_cast<char *>(out);
    a.lse = lse;
    a.partial = static_cast<float *>(workspace);
    const unsigned grid = attention::spread(a, work, (int64_t)a.row_tiles * a.splits);
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    if (!attention::allow_lds(reinterpret_cast<const void *>(v.kernel), v.lds))
        return GRKAN_ERR_LAUNCH;
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3(grid), dim3(256), args, v.lds, stream) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    if (a.splits > 1) {
        const int64_t lanes = (int64_t)a.batch * a.kv_heads * a.rows * (a.dim / 8), blocks = (lanes + 255) / 256;
        if (blocks > INT32_MAX)
            return GRKAN_ERR_UNSUPPORTED;
        if (io == GRKAN_BF16)
            attention::join_kernel<__bf16><<<dim3((unsigned)blocks), 256, 0, stream>>>(a);
        else
            attention::join_kernel<_Float16><<<dim3((unsigned)blocks), 256, 0, stream>>>(a);
        if (hipGetLastError() != hipSuccess)
            return GRKAN_ERR_LAUNCH;
    }
    return GRKAN_OK;
}
