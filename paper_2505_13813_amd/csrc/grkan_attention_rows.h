// What the forward kernels of attention share: 32 rows of a wavefront on their way through the keys, and the joining of parts.
#ifndef GRKAN_ATTENTION_ROWS_H_
#define GRKAN_ATTENTION_ROWS_H_

#include "grkan_attention.h"

namespace grkan {
namespace attention {

// 32 rows of a wavefront: their queries, the running maximum and sum, and the sum of the weighted values.
template <typename IO, int DP, int KT> struct Rows {
    typedef IO Type;
    using MM = Matrix<IO>;
    static constexpr int KB = KT / 32, ND = DP / 32, NS = DP / 16;
    static constexpr uint64_t kAll = KT == 64 ? ~(uint64_t)0 : 0xffffffffu;

    u32x4 q[NS];   // second operands: lane l has row l mod 32, channels 16 s + 8 (l / 32) ..
    f32x16 acc[ND]; // lane l has channels 32 d + 8 (i / 4) + 4 (l / 32) + i mod 4 of row l mod 32
    float top, sum; // the maximum that the probabilities are relative to; this lane's part of their sum

    __device__ __forceinline__ void load(const Args &a, int32_t b, int32_t kvh, uint32_t row, uint32_t h)
    {
        load(a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head + row_offset(row, (uint32_t)a.group, a.q.token, a.q.head)),
             (int64_t)row < a.rows, a.dim, h);
    }
    // the row at that address, or zeros
    __device__ __forceinline__ void load(uint64_t at, bool row_there, int32_t dim, uint32_t h)
    {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool there = row_there && channel < (uint32_t)dim;
            q[s] = gload16(there ? at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int d = 0; d < ND; ++d)
            acc[d] = f32x16{};
        top = -__builtin_inff();
        sum = 0.0f;
    }

    // One tile of keys.  word: which of them are valid, and cover what write_cover left of that, where it is not all; c: of the scores, in powers
    // of 2
    __device__ __forceinline__ void take(const Addresses<NS> &k_from, const Addresses<ND> &v_from, uint64_t word, uint32_t cover, float c, uint32_t h)
    {
        f32x16 s[KB];
        if (word != kAll) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                s[kb] = read_cover(cover, kb, h);
#pragma unroll
            for (int st = 0; st < NS; ++st)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    s[kb] = MM::multiply(RowOperand<DP>::read(k_from, kb, st), q[st], s[kb]);
        } else {
            scores(k_from, s);
        }
        uint32_t p[KB][8];
        probabilities(s, c, p);
        add(p, v_from);
    }

    // The scores without a mask.
    __device__ __forceinline__ void scores(const Addresses<NS> &k_from, f32x16 (&s)[KB])
    {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            s[kb] = f32x16{};
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                s[kb] = MM::multiply(RowOperand<DP>::read(k_from, kb, st), q[st], s[kb]);
    }

    // As scores, with the operands of AHEAD products read in front of the one that is computed.
    template <int AHEAD> __device__ __forceinline__ void scores_ahead(const Addresses<NS> &k_from, f32x16 (&s)[KB])
    {
        scores(k_from, s);
        __builtin_amdgcn_sched_group_barrier(kLdsReads, AHEAD * KB, 0);
#pragma unroll
        for (int st = AHEAD; st < NS; ++st) {
            __builtin_amdgcn_sched_group_barrier(kProducts, KB, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, KB, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, AHEAD * KB, 0);
    }

    // Keys behind `last` (of the tile, the lane's row's last valid one; below 0: none) are not valid.
    static __device__ __forceinline__ void cut(f32x16 (&s)[KB], int32_t last, uint32_t h)
    {
        last -= 4 * (int32_t)h;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[kb][i] = 32 * kb + 8 * (i / 4) + i % 4 <= last ? s[kb][i] : -__builtin_inff();
    }

    // scores to probabilities, in the order of the product's operand; the statistics, and the sums so far, move along
    __device__ __forceinline__ void probabilities(const f32x16 (&s)[KB], float c, uint32_t (&p)[KB][8])
    {
        float most = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                most = fmaxf(most, s[kb][i]);
        most = halves_max(most);
        if (__ballot(most > top + fminf(8.0f / c, 1e38f)) != 0) {
            const float next = fmaxf(top, most);
            const float by = next > -__builtin_inff() ? __builtin_amdgcn_exp2f((top - next) * c) : 1.0f;
            sum *= by;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[d][i] *= by;
            top = next;
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
    }

    static __device__ __forceinline__ u32x4 operand(const uint32_t (&p)[8], int t)
    {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = p[4 * t + j];
        return w;
    }

    __device__ __forceinline__ void add(const uint32_t (&p)[KB][8], const Addresses<ND> &v_from)
    {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u32x4 w = operand(p[kb], t);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    acc[d] = MM::multiply(ColumnOperand<DP>::read(v_from, kb, t, d), w, acc[d]);
            }
    }

    // scores of a tile and add of another, in the order that is written: operands are read four products ahead, and between(n), n from 0 to
    // 3, goes between the products.
    template <class Between>
    __device__ __forceinline__ void scores_and_add(const Addresses<NS> &k_from, f32x16 (&s)[KB], const uint32_t (&p)[KB][8], const Addresses<ND> &v_from, Between &&between)
    {
        constexpr int kScores = NS * KB, kAll = kScores + 2 * KB * ND, kAhead = 4;
        auto operand = [&](int n) {
            const int i = n - kScores;
            return n < kScores ? RowOperand<DP>::read(k_from, n % KB, n / KB) : ColumnOperand<DP>::read(v_from, i / (2 * ND), i / ND % 2, i % ND);
        };
        u32x4 next[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n)
            next[n] = operand(n);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            s[kb] = f32x16{};
#pragma unroll
        for (int n = 0; n < kAll; ++n) {
            const int i = n - kScores;
            if (n < kScores)
                s[n % KB] = MM::multiply(next[n % kAhead], q[n / KB], s[n % KB]);
            else
                acc[i % ND] = MM::multiply(next[n % kAhead], this->operand(p[i / (2 * ND)], i / ND % 2), acc[i % ND]);
            if (n + kAhead < kAll)
                next[n % kAhead] = operand(n + kAhead);
            if (n % (kAll / 4) == kAll / 8)
                between(n / (kAll / 4));
            fence_schedule();
        }
    }

    // As add, for scores that were cut: a row at a time, with zeros in place of the values behind its last key.  (Zero times a NaN or an infinity
    // is NaN, so the rows of one product must not differ in what they may see where a value is one.)
    __device__ __forceinline__ void add_each(const uint32_t (&p)[KB][8], const Addresses<ND> &v_from, int32_t last, uint32_t col, uint32_t h)
    {
#pragma unroll 1
        for (uint32_t r = 0; r < 32; ++r) {
            const int32_t mine = __builtin_amdgcn_readlane(last, (int)r) - 4 * (int32_t)h;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 w = operand(p[kb], t);
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        fence_schedule(); // (one at a time: it is rare, and has few registers)
                        u32x4 v = ColumnOperand<DP>::read(v_from, kb, t, d);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int32_t key = 32 * kb + 16 * t + 8 * (j / 2) + 2 * (j % 2);
                            v[j] = key > mine ? 0u : key + 1 > mine ? v[j] & 0xffffu : v[j];
                        }
                        const f32x16 all = MM::multiply(v, w, acc[d]);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            acc[d][i] = col == r ? all[i] : acc[d][i];
                    }
                }
        }
    }

    // Whether a sum of any row is a NaN or an infinity.
    __device__ __forceinline__ bool not_finite() const
    {
        float x = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x = fmaf(acc[d][i], 0.0f, x);
        return __ballot(x != x) != 0;
    }
};

// Channels 32 d .. of a row, as the sums lie in the lanes: of the output, or as they are to a row of float32
template <typename IO> __device__ __forceinline__ void store_channels(const f32x16 &sums, int d, float by, const Args &a, char *out, bool wide, uint32_t h)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int channel = 32 * d + 8 * g + 4 * (int)h;
        if (channel >= a.dim)
            continue;
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            o[j] = sums[4 * g + j] * by;
        if (wide) {
            *reinterpret_cast<f32x4 *>(out + channel * 4) = o;
        } else {
            u32x2 w;
            w[0] = Matrix<IO>::two(o[0], o[1]);
            w[1] = Matrix<IO>::two(o[2], o[3]);
            *reinterpret_cast<u32x2 *>(out + channel * 2) = w;
        }
    }
}

// Where row r of a key head goes in the output.
__device__ __forceinline__ char *out_row(const Args &a, int32_t b, int32_t kvh, uint32_t row)
{
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    return a.out + 2 * ((int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim +
                        row_offset(row, (uint32_t)a.group, heads_dim, a.dim));
}

// log2 of a row's sum as the splits keep it; the caller's lse has an infinity for a row without a valid key
__device__ __forceinline__ float log2_sum(float top, float sum, float c)
{
    return sum == 0.0f ? -__builtin_inff() : top * c + __builtin_amdgcn_logf(sum);
}
__device__ __forceinline__ float lse_of(float l2) { return l2 == -__builtin_inff() ? __builtin_inff() : l2; }

// ------------------------------------------------------------------------------------------------ four wavefronts on the keys of 32 rows

template <typename IO_, int DP_> struct TokenShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, KT = 32, kWaves = 4;
    static constexpr uint32_t kTile = kTileBytes<DP, KT>, kStage = 2 * kTile;
    static constexpr uint32_t kCover = kStage * 2 * kWaves; // behind the tiles, two of each wavefront
    static constexpr size_t kLds = kCover + 2 * KT * 4 * kWaves;
    static_assert(kGroup % (KT * kWaves) == 0, "");
    static_assert(((DP + 4) * 32 * kWaves + 64 * kWaves) * sizeof(float) <= kLds, ""); // what the wavefronts join
};

// A wavefront's way through tiles t0, t0 + kWaves, .. (t0 its own first), below t1, without a barrier: the loads of the next are in flight
// while one is computed with.  word_of(t): which keys of a tile are valid (asked in rising order); load(t, word, whole, to): K of the tile
// to `to`, V behind it.  Returns whether there was a valid key. (Each part of the loop is in the code once, the first tile's loads too.)
template <class SH, class Word, class Load>
__device__ __forceinline__ bool walk_alone(Rows<typename SH::IO, SH::DP, SH::KT> &rows, int32_t t0, int32_t t1, uint32_t lds0, int wave, int lane, float c,
                                           int32_t dim, Word &&word_of, Load &&load)
{
    constexpr int DP = SH::DP, KT = SH::KT, kStep = SH::kWaves;
    constexpr int kAhead = 2 * TileLoads<DP, KT, 1>::kMine;
    const RowOperand<DP> k_operand(lane);
    const ColumnOperand<DP> v_operand(lane);
    const uint32_t h = (uint32_t)lane >> 5;
    const uint32_t stages = lds0 + (uint32_t)wave * 2u * SH::kStage, covers = lds0 + SH::kCover + (uint32_t)wave * 2u * KT * 4u;
    arrived(rows.q);
    uint32_t at = SH::kStage;
    uint64_t word = 0, some = 0; // valid keys: of a tile, of any
#pragma unroll 1
    for (int32_t t = t0 - kStep; t < t1; t += kStep) {
        const bool more = t + kStep < t1;
        const uint64_t next = more ? word_of(t + kStep) : 0;
        if (more) {
            load(t + kStep, next, next == rows.kAll && dim == DP, stages + (at ^ SH::kStage));
            if (next != rows.kAll && lane < KT)
                write_cover(covers + (at ? 0u : KT * 4u), next, lane);
        }
        if (t >= t0) {
            if (more)
                wait_loads<kAhead>();
            else
                wait_loads<0>();
            rows.take(k_operand.moved(stages + at), v_operand.moved(stages + at + SH::kTile), word, covers + (at ? KT * 4u : 0u), c, h);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (the tile's buffer is loaded into next)
        }
        at ^= SH::kStage;
        some |= word;
        word = next;
    }
    return some != 0;
}

// The wavefronts' parts of each row: sums relative to a common maximum, added in wavefront order.  out, lse: the lane's row's; wide: as
// parts to be joined are kept.
template <class SH>
__device__ __forceinline__ void join_wavefronts(const Rows<typename SH::IO, SH::DP, SH::KT> &rows, char *smem, int wave, int lane, bool there, const Args &a, char *out,
                                                float *lse, bool wide)
{
    constexpr int DP = SH::DP, ND = DP / 32;
    constexpr int kPitch = DP + 4; // of a row's channels
    const uint32_t row = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    const float c = a.c;
    float *const joined = reinterpret_cast<float *>(smem);  // [wave][32 rows][channel]
    float *const stats = joined + SH::kWaves * 32 * kPitch; // [wave][2][32 rows]
    const float mine = halves_sum(rows.sum);
    wait_loads<0>();
    barrier();
    if (h == 0) {
        stats[wave * 64 + row] = rows.top;
        stats[wave * 64 + 32 + row] = mine;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[j] = rows.acc[d][4 * g + j];
            *reinterpret_cast<f32x4 *>(joined + (wave * 32 + (int)row) * kPitch + 32 * d + 8 * g + 4 * (int)h) = o;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    float top = -__builtin_inff(), sum = 0.0f, by[SH::kWaves];
#pragma unroll
    for (int w = 0; w < SH::kWaves; ++w)
        top = fmaxf(top, stats[w * 64 + row]);
#pragma unroll
    for (int w = 0; w < SH::kWaves; ++w) {
        const float m = stats[w * 64 + row];
        by[w] = m > -__builtin_inff() ? __builtin_amdgcn_exp2f((m - top) * c) : 0.0f;
        sum += stats[w * 64 + 32 + row] * by[w];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum, l2 = log2_sum(top, sum, c);
    if (there) { // wavefront w writes channels 32 w .., 32 (w + kWaves) ..
#pragma unroll 1
        for (int d = wave; d < ND; d += SH::kWaves) {
            f32x16 all;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 o = {};
#pragma unroll
                for (int w = 0; w < SH::kWaves; ++w) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(joined + (w * 32 + (int)row) * kPitch + 32 * d + 8 * g + 4 * (int)h);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        o[j] += x[j] * by[w];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    all[4 * g + j] = o[j];
            }
            store_channels<typename SH::IO>(all, d, inv, a, out, wide, h);
        }
        if (h == 0 && wave == 0) {
            if (wide)
                *lse = l2;
            else if (a.lse)
                *lse = lse_of(l2);
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier(); // (the next part's tiles come where the joined rows were)
}

// A row's parts p of `parts`, each the mean over its own keys, by the share of the sum that each has: eight channels of it, rounded to
// `out`, and the row's lse. values(p), stats(p): a part's channels and log2 of its sum.  `lanes` adjacent lanes, of which this is number
// `lane`, have every lanes-th part each and then add up; the first writes.  Eight parts' loads are out at once: it is their latency that
// all this takes (23 parts of twelve key heads with 64 channels and two rows: 10.2 us with a lane for all parts, 6.0 with sixteen).
template <typename IO, typename Values, typename Stats>
__device__ __forceinline__ float join_parts(int32_t parts, int32_t lane, int32_t lanes, Values &&values, Stats &&stats, char *out)
{
    float most = -__builtin_inff(), total = 0.0f, o[8] = {};
    // (a part without a valid key has a share of 0 and a row of zeros)
    auto share_of = [](float l2, float top) { return __builtin_amdgcn_exp2f(l2 - (top == -__builtin_inff() ? 0.0f : top)); };
    // parts p0, p0 + lanes, .., COUNT of them but those behind the last
    auto take = [&](auto count, int32_t p0) {
        constexpr int COUNT = decltype(count)::value;
        f32x4 x[COUNT], y[COUNT];
        float l2[COUNT], top = most;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) {
            const int32_t p = p0 + j * lanes < parts ? p0 + j * lanes : parts - 1;
            const f32x4 *const from = reinterpret_cast<const f32x4 *>(values(p));
            x[j] = from[0];
            y[j] = from[1];
            l2[j] = stats(p);
        }
#pragma unroll
        for (int j = 0; j < COUNT; ++j) {
            l2[j] = p0 + j * lanes < parts ? l2[j] : -__builtin_inff();
            top = fmaxf(top, l2[j]);
        }
        const float by = share_of(most, top);
        most = top;
        total *= by;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            o[i] *= by;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) {
            const float share = share_of(l2[j], top);
            total += share;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] += share * x[j][i];
                o[4 + i] += share * y[j][i];
            }
        }
    };
#pragma unroll 1
    for (int32_t p = 0; p < parts;) {
        if (parts - p > 2 * lanes) {
            take(std::integral_constant<int, 8>{}, p + lane);
            p += 8 * lanes;
        } else {
            take(std::integral_constant<int, 2>{}, p + lane);
            p += 2 * lanes;
        }
    }
    for (int32_t s = 1; s < lanes; s *= 2) {
        const float other = __shfl_xor(most, s), top = fmaxf(most, other), by = share_of(most, top), by_other = share_of(other, top);
        most = top;
        total = total * by + __shfl_xor(total, s) * by_other;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            o[i] = o[i] * by + __shfl_xor(o[i], s) * by_other;
    }
    if (lane == 0) {
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = Matrix<IO>::two(o[2 * j] * inv, o[2 * j + 1] * inv);
        *reinterpret_cast<u32x4 *>(out) = w;
    }
    return total == 0.0f ? __builtin_inff() : most + __builtin_amdgcn_logf(total);
}

} // namespace attention
} // namespace grkan
#endif // GRKAN_ATTENTION_ROWS_H_
