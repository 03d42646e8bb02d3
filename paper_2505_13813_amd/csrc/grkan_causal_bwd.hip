// Causal attention over packed sequences on gfx950 (MI355X), backward.  With P recomputed from the rows' lse, D = dO V^T and delta = the
// row's sum of dO O, of what out was before it was rounded (out and the rest: an error of delta goes into all of a row's S', and with out
// alone it is a third of the gradients' own rounding in a sequence of 60 tokens),
//
//     dV_j = sum_{i >= j} P_ij dO_i      S'_ij = P_ij (D_ij - delta_i)      dQ_i = scale sum_{j <= i} S'_ij K_j      dK_j = scale sum_{i >= j} S'_ij Q_i
//
// in two kernels as cross attention has them (grkan_attention_bwd.hip): one owns keys and walks the rows that see them, one owns rows and
// walks the keys that they see; no atomics, the same bits each time.  Tiles that the diagonal crosses take comparisons, the others none,
// and what lies behind it is left out.
//
// A key sees the more rows the earlier it is, so the walks of a long sequence's first keys are cut into slabs of rows, each a workgroup's,
// whose sums a second launch adds up; the queries' kernel starts its longest walks first.
//
// What bounds it: products and vector operations, as of the forward pass (by the profiler, whose times are 6 to 13 % above those of calls in a
// row: 4,001 and 2,852 tokens, 16 heads of 128 on four: queries 174 us, keys 255, 0.85 and 0.78 PFLOP/s; sixteen sequences of 90 to 1,500
// tokens, twelve heads of 64: 36 and 42 us, and 8 for the slabs' sums; the same in float16, with 17 and 9 us for the rows in front: 173 and
// 282; 32, 48 and 8).
//
// float16: scaled as there; the largest upstream gradient is that of the key's own sequence, from the key's tile on.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "grkan_attention_back.h"
#include "grkan_packed.h"

namespace grkan {
namespace attention {

// float16: of 64 rows of a segment delta, and the largest |dO| and |delta|: sixteen lanes a row, eight channels each.
template <typename IO> __global__ __launch_bounds__(256) void causal_rows_kernel(const Packed a)
{
    using MM = Matrix<IO>;
    __shared__ uint32_t most[4][2];
    const int32_t slot = (int32_t)blockIdx.x / a.kv_heads, kvh = (int32_t)blockIdx.x - slot * a.kv_heads;
    const Segment s = segment_of<kRowTile>(a, slot, a.group, true);
    const int32_t all = s.count * a.group;
    if (s.none || (int64_t)s.tile * kRowTile >= all)
        return;
    const uint32_t lane16 = threadIdx.x & 15u;
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    const uint64_t out = a.forward_out + (uint64_t)packed_at(a, s, kvh, 0), rest = reinterpret_cast<uint64_t>(a.rest) + (uint64_t)packed_at(a, s, kvh, 0);
    const uint64_t dout = a.dout.at + (uint64_t)((int64_t)s.first * a.dout.token + (int64_t)kvh * a.group * a.dout.head);
    const uint32_t row0 = (uint32_t)s.tile * kRowTile + (threadIdx.x >> 4);
    u32x4 o[4], d[4], left[4];
    float largest = 0.0f, sums = 0.0f;
    // (all loads in front, without a branch: they wait for one another otherwise)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t row = row0 + 16u * k;
        const bool there = (int32_t)row < all, loaded = there && 8u * lane16 < (uint32_t)a.dim;
        const uint64_t zeros = reinterpret_cast<uint64_t>(kZeros);
        const uint64_t at = 2u * (uint64_t)row_offset(row, (uint32_t)a.group, heads_dim, a.dim) + 16u * lane16;
        o[k] = gload16(loaded ? out + at : zeros, 0);
        left[k] = gload16(loaded && a.rest ? rest + at : zeros, 0);
        d[k] = gload16(loaded ? dout + (uint64_t)row_offset(row, (uint32_t)a.group, a.dout.token, a.dout.head) + 16u * lane16 : zeros, 0);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t row = row0 + 16u * k;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = MM::first(d[k][j]), y = MM::second(d[k][j]);
            sum += x * (MM::first(o[k][j]) + MM::first(left[k][j])) + y * (MM::second(o[k][j]) + MM::second(left[k][j]));
            largest = fmaxf(largest, fmaxf(fabsf(x), fabsf(y)));
        }
#pragma unroll
        for (int i = 8; i > 0; i /= 2)
            sum += __shfl_xor(sum, i);
        sums = fmaxf(sums, fabsf(sum));
        if (lane16 == 0 && (int32_t)row < all)
            a.row_delta[(int64_t)kvh * a.rows + packed_row(a, s, row)] = sum;
    }
    const uint32_t bits[2] = {most_of_lanes(__builtin_bit_cast(uint32_t, largest)), most_of_lanes(__builtin_bit_cast(uint32_t, sums))};
    if ((threadIdx.x & 63) == 0) {
        most[threadIdx.x >> 6][0] = bits[0];
        most[threadIdx.x >> 6][1] = bits[1];
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        uint32_t found = 0;
        for (int w = 0; w < 4; ++w)
            found = most[w][threadIdx.x] > found ? most[w][threadIdx.x] : found;
        a.row_most[2 * ((int64_t)kvh * a.row_tiles + place_of<kRowTile>(s.first, a.group, s.index) + s.tile) + threadIdx.x] = __builtin_bit_cast(float, found);
    }
}

// PARTS: wavefronts that share the rows of a stage, for the same 32 keys, or the keys of a tile, for the same 32 rows; the others have keys
// or rows of their own.
template <typename IO, int DP, int ROWS, bool V_LDS, int PER, int PARTS_, bool FINE_> struct CausalBackShape : BackShape<IO, DP, ROWS, V_LDS, PER> {
    using Base = BackShape<IO, DP, ROWS, V_LDS, PER>;
    static constexpr bool FINE = FINE_;
    static constexpr int PARTS = PARTS_, kOwn = 32 * Base::kWaves / PARTS;
    static constexpr uint32_t kValues = V_LDS ? kOwn / 64 * Base::kKeysTile : 0; // in front of the stages
    static constexpr size_t kKeyLds = 2 * (size_t)Base::kKeyStage + kValues;
    static_assert(PARTS == 1 || (ROWS == 64 && (size_t)2 * 2 * (DP / 8) * 64 * 16 <= kKeyLds), ""); // what the wavefronts join
};

// The rows that tile `tile` of a segment's keys is seen by: tiles [first, tiles) of `size` rows, in `parts` slabs of `per`, the first of
// what remains.
struct Walk {
    int32_t first, tiles, parts, per;
    __device__ __forceinline__ int32_t begin(int32_t part) const { return part == 0 ? first : tiles - (parts - part) * per; }
    __device__ __forceinline__ Walk(const Packed &a, const Segment &s, int32_t own, int32_t size)
    {
        const int32_t all = s.count * a.group;
        first = (int32_t)((int64_t)s.tile * own * a.group / size);
        tiles = (all + size - 1) / size;
        const int32_t n = tiles - first, most = (n + a.parts - 1) / a.parts;
        per = a.slab > most ? a.slab : most;
        parts = n > per ? (n + per - 1) / per : 1;
    }
};

// Sums of two wavefronts of the same keys or rows: the second leaves its own in LDS (and is done: false), the first adds them.
template <int N, typename Sums> __device__ __forceinline__ bool add_second(char *smem, int own, int shared, int lane, Sums &&sums)
{
    f32x4 *const place = reinterpret_cast<f32x4 *>(smem) + own * N * 4 * 64 + lane;
    wait_loads<0>();
    barrier(); // (all are done with what lay there)
    if (shared == 1) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[j] = sums(n)[4 * g + j];
                place[(4 * n + g) * 64] = o;
            }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    if (shared == 1)
        return false;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 o = place[(4 * n + g) * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sums(n)[4 * g + j] += o[j];
        }
    return true;
}

// What rounding x and y to w took away.  FINE: S' goes into the products in two parts of 16 bits.  Rounded once, its error is as large as
// that of the gradients' own rounding: dQ and dK are off by 1.41 to 1.47 times that, in sequences of some dozen tokens by up to 1.51; with
// two parts by 1.02 to 1.09.
template <class MM> __device__ __forceinline__ uint32_t rest_of(uint32_t w, float x, float y) { return MM::two(x - MM::first(w), y - MM::second(w)); }

// dK and dV of 32 keys a wavefront, from all the rows that see them or a slab of those.  Whole slabs are launched first, what remains of a
// walk last.
template <class SH> __global__ __launch_bounds__(256, SH::PER) void causal_keys_kernel(const Packed a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, ROWS = SH::ROWS, ND = DP / 32, NS = DP / 16;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    // block ((part, slot), key head)
    const int32_t turn = (int32_t)blockIdx.x / a.kv_heads, kvh = (int32_t)blockIdx.x - turn * a.kv_heads;
    const int32_t back = turn / a.key_tiles, part = a.parts - 1 - back, slot = turn - back * a.key_tiles;
    const int own = wave / SH::PARTS, shared = wave % SH::PARTS;
    const Segment s = segment_of<SH::kOwn>(a, slot, 1, false);
    const int64_t begin = (int64_t)s.tile * SH::kOwn;
    if (begin >= s.count)
        return;
    const Walk walk(a, s, SH::kOwn, ROWS);
    if (part >= (s.none ? 1 : walk.parts))
        return;
    const int32_t all = s.count * a.group, count = s.count;
    const int32_t t0 = walk.begin(part), t1 = s.none ? t0 : part + 1 < walk.parts ? walk.begin(part + 1) : walk.tiles;
    const int32_t key0 = (int32_t)begin + own * 32, key = key0 + (int32_t)col; // this wavefront's and this lane's
    const bool valid = key < count, works = key0 < count;

    // ---- keys and values as second operands: lane l has key l mod 32, channels 16 s + 8 (l / 32) ..
    u32x4 k[NS], v[SH::V_LDS ? 1 : NS];
    const uint64_t k_base = a.k.at + (uint64_t)((int64_t)s.first * a.k.token + kvh * a.k.head);
    const uint64_t v_base = a.v.at + (uint64_t)((int64_t)s.first * a.v.token + kvh * a.v.head);
#pragma unroll
    for (int st = 0; st < NS; ++st) {
        const uint32_t channel = 16u * st + 8u * h;
        const bool there = valid && channel < (uint32_t)a.dim;
        k[st] = gload16(there ? k_base + (uint64_t)key * (uint64_t)a.k.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        if constexpr (!SH::V_LDS)
            v[st] = gload16(there ? v_base + (uint64_t)key * (uint64_t)a.v.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
    }
    f32x16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        dk[d] = f32x16{};
        dv[d] = f32x16{};
    }

    const uint64_t q_base = a.q.at + (uint64_t)((int64_t)s.first * a.q.token + (int64_t)kvh * a.group * a.q.head);
    const uint64_t d_base = a.dout.at + (uint64_t)((int64_t)s.first * a.dout.token + (int64_t)kvh * a.group * a.dout.head);
    const RowsTwiceLoads<DP, ROWS, SH::kWaves> q_loads(wave, lane, a.q, a), d_loads(wave, lane, a.dout, a);
    const float c = a.c;
    float up = 1.0f; // of the key
    if constexpr (kRowsFirst<IO>) {
        u32x4 value[NS];
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            const uint32_t channel = 16u * st + 8u * h;
            const bool there = valid && channel < (uint32_t)a.dim;
            value[st] = gload16(there ? v_base + (uint64_t)key * (uint64_t)a.v.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
        const int32_t base = place_of<kRowTile>(s.first, a.group, s.index);
        const int32_t row_tiles = s.none ? 0 : (all + kRowTile - 1) / kRowTile;
        uint32_t largest = 0, sums = 0;
        for (int32_t i = (int32_t)(begin * a.group / kRowTile) + lane; i < row_tiles; i += 64) {
            const f32x2 both = reinterpret_cast<const f32x2 *>(a.row_most)[(int64_t)kvh * a.row_tiles + base + i];
            largest = greater(largest, both[0]);
            sums = greater(sums, both[1]);
        }
        float length2 = 0.0f;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                length2 += MM::first(value[st][j]) * MM::first(value[st][j]) + MM::second(value[st][j]) * MM::second(value[st][j]);
        length2 = halves_sum(length2);
        up = lowered(scale_of(most_of_lanes(largest)), length2, __builtin_bit_cast(float, most_of_lanes(sums)), a.dim);
        const uint32_t longest = most_of_lanes(__builtin_bit_cast(uint32_t, length2) & 0x7fffffffu);
        if (lane == 0 && part == 0 && shared == 0)
            a.value_most[((int64_t)kvh * a.value_tiles + place_of<kGroup>(s.first, 1, s.index)) * (kGroup / 32) + key0 / 32] = __builtin_bit_cast(float, longest);
    }

    auto issue = [&](int32_t t, uint32_t stage) {
        q_loads.issue(a.q, q_base, t, all, a, stage);
        d_loads.issue(a.dout, d_base, t, all, a, stage + SH::kRowsTile);
        if (wave < 2) {
            const float *const from = (wave ? a.row_delta : a.lse) + (int64_t)kvh * a.rows + packed_row(a, s, (int64_t)t * ROWS);
            const int32_t l = (int32_t)lane_here(), left = all - t * ROWS;
            if (l < ROWS)
                load_words_to_lds(uniform_u64(reinterpret_cast<uint64_t>(from)), (uint32_t)(l < left ? l : left - 1) * 4u,
                                  stage + 2 * SH::kRowsTile + (uint32_t)wave * ROWS * 4u);
        }
    };

    const uint32_t stages = lds0 + SH::kValues;
    // (moved from stage to stage in place: there are no registers for copies)
    RowOperand<DP> rows(lane), v_rows(lane);
    ColumnOperand<DP> columns(lane);
    rows.move(stages + SH::kKeyStage + row_at<DP>((uint32_t)(32 * shared)));
    columns.move(stages + SH::kKeyStage + row_at<DP>((uint32_t)(32 * shared)));
    v_rows.move(lds0 + (uint32_t)own * row_at<DP>(32u));
    uint32_t at = SH::kKeyStage;
    if constexpr (SH::V_LDS) {
        if (t0 < t1) {
            const TileLoads<DP, 64, SH::kWaves> v_loads(wave, lane, a.v.token, a.dim);
#pragma unroll 1
            for (int half = 0; half < SH::kOwn / 64; ++half) {
                const int32_t first = (int32_t)begin + 64 * half;
                v_loads.issue(v_base + (uint64_t)first * (uint64_t)a.v.token, a.v.token, __ballot(first + lane < count), false, lds0 + (uint32_t)half * SH::kKeysTile);
            }
        }
    }
    if (a.dim < DP) {
#pragma unroll 1
        for (uint32_t stage = stages; stage < stages + 2 * SH::kKeyStage; stage += SH::kKeyStage) {
            q_loads.clear(lane, stage);
            d_loads.clear(lane, stage + SH::kRowsTile);
        }
    }
    arrived(k);
    if constexpr (!SH::V_LDS)
        arrived(v);
    const int32_t first_row = key0 * a.group, last_row = (key0 + 31) * a.group; // that see the wavefront's first key, and its last
#pragma unroll 1
    for (int32_t t = t0 - 1; t < t1; ++t) {
        if (t >= t0) {
            wait_loads<0>();
            barrier();
        }
        if (t + 1 < t1)
            issue(t + 1, stages + (at ^ SH::kKeyStage));
        const uint32_t by = at ? SH::kKeyStage : 0u - SH::kKeyStage, stage = stages + at;
        at ^= SH::kKeyStage;
        if (t >= t0) {
            rows.move(by);
            columns.move(by);
        }
        if (t < t0 || !works || (t + 1) * ROWS <= first_row)
            continue;
        const uint32_t stats = stage + 2 * SH::kRowsTile + 128u * (uint32_t)shared + 16u * (lane_here() >> 5);
        const bool crossed = t * ROWS < last_row || (t + 1) * ROWS > all;
#pragma unroll
        for (int rb = 0; rb < ROWS / 32 / SH::PARTS; ++rb) {
            f32x16 p = {}, d = {};
            // (both at once, in the order that is written, and operands read two steps ahead: each product waits for its own LDS reads
            // otherwise, for four times its own time)
            {
                constexpr int kAhead = 2;
                u32x4 x[kAhead], y[kAhead], z[kAhead];
                auto read = [&](int st) {
                    x[st % kAhead] = RowOperand<DP>::read(rows, rb, st);
                    y[st % kAhead] = RowOperand<DP>::read(rows, rb, st, SH::kRowsTile);
                    if constexpr (SH::V_LDS)
                        z[st % kAhead] = RowOperand<DP>::read(v_rows, 0, st);
                    else
                        z[st % kAhead] = v[st];
                };
#pragma unroll
                for (int st = 0; st < kAhead; ++st)
                    read(st);
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    p = MM::multiply(x[st % kAhead], k[st], p);
                    d = MM::multiply(y[st % kAhead], z[st % kAhead], d);
                    if (st + kAhead < NS)
                        read(st + kAhead);
                    fence_schedule();
                }
            }
            u32x4 w[2], left[2];
#pragma unroll
            for (int quad = 0; quad < 4; ++quad) {
                const f32x4 lse = __builtin_bit_cast(f32x4, lds_read16(stats + (32u * rb + 8u * quad) * 4u));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    p[4 * quad + j] = __builtin_amdgcn_exp2f(fmaf(p[4 * quad + j], c, -lse[j]));
            }
            if (crossed) { // rows of the tile that see the key: from `from` on, and before the segment's end
                const int32_t l = (int32_t)lane_here(), row0 = t * ROWS + 32 * (rb + shared) + 4 * (l >> 5);
                const int32_t from = (key0 + (l & 31)) * a.group - row0;
                const uint32_t span = (uint32_t)(all - row0 - from);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    p[i] = (uint32_t)(8 * (i / 4) + i % 4 - from) < span ? p[i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                w[i / 4][i % 4] = MM::two(p[2 * i], p[2 * i + 1]);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int n = 0; n < ND; ++n)
                    dv[n] = MM::multiply(ColumnOperand<DP>::read(columns, rb, half, n, SH::kRowsTile), w[half], dv[n]);
#pragma unroll
            for (int quad = 0; quad < 4; ++quad) {
                const f32x4 delta = __builtin_bit_cast(f32x4, lds_read16(stats + (ROWS + 32u * rb + 8u * quad) * 4u));
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = p[4 * quad + j] * fmaf(d[4 * quad + j], up, -delta[j] * up);
                w[quad / 2][2 * (quad % 2)] = MM::two(y[0], y[1]);
                w[quad / 2][2 * (quad % 2) + 1] = MM::two(y[2], y[3]);
                if constexpr (SH::FINE) {
                    left[quad / 2][2 * (quad % 2)] = rest_of<MM>(w[quad / 2][2 * (quad % 2)], y[0], y[1]);
                    left[quad / 2][2 * (quad % 2) + 1] = rest_of<MM>(w[quad / 2][2 * (quad % 2) + 1], y[2], y[3]);
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int n = 0; n < ND; ++n) {
                    const u32x4 column = ColumnOperand<DP>::read(columns, rb, half, n);
                    dk[n] = MM::multiply(column, w[half], dk[n]);
                    if constexpr (SH::FINE)
                        dk[n] = MM::multiply(column, left[half], dk[n]);
                }
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 8, 0);
#pragma unroll
            for (int n = 0; n < 2 * ND; ++n) {
                __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
            }
#pragma unroll
            for (int n = 4; n < 2 * ND; ++n) {
                __builtin_amdgcn_sched_group_barrier(kProducts, SH::FINE ? 2 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 4, 0);
            __builtin_amdgcn_sched_group_barrier(kProducts, SH::FINE ? 8 : 4, 0);
        }
    }

    if constexpr (SH::PARTS > 1) // the first adds what the second has
        if (!add_second<2 * ND>(smem, own, shared, lane, [&](int n) -> f32x16 & { return n < ND ? dk[n] : dv[n - ND]; }))
            return;
    const int32_t l = (int32_t)lane_here(), mine = key0 + (l & 31);
    if (mine >= count)
        return;
    const float by = a.scale / up;
    const int64_t line = ((int64_t)s.first + mine) * a.kv_heads + kvh;
    const bool whole = s.none || walk.parts == 1;
    // parts: [slab][dK, dV][tokens, kv_heads, dim]
    const int64_t lines = (int64_t)a.tokens * a.kv_heads;
    float *const to = a.partial + (2 * part * lines + line) * a.dim;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int channel = 32 * n + 8 * g + 4 * (l >> 5);
            if (channel >= a.dim)
                continue;
            f32x4 x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = dk[n][4 * g + j] * by;
                y[j] = dv[n][4 * g + j];
            }
            if (whole) {
                u32x2 u, z;
                u[0] = MM::two(x[0], x[1]);
                u[1] = MM::two(x[2], x[3]);
                z[0] = MM::two(y[0], y[1]);
                z[1] = MM::two(y[2], y[3]);
                *reinterpret_cast<u32x2 *>(a.dk + (line * a.dim + channel) * 2) = u;
                *reinterpret_cast<u32x2 *>(a.dv + (line * a.dim + channel) * 2) = z;
            } else {
                *reinterpret_cast<f32x4 *>(to + channel) = x;
                *reinterpret_cast<f32x4 *>(to + lines * a.dim + channel) = y;
            }
        }
}

// The sum of the slabs' parts of a tile of keys, in their order: block (slot, key head), or four of them, one for each half of the keys and each of
// dK and dV; four times four elements a lane and pass.
template <typename IO, int OWN> __global__ __launch_bounds__(256) void causal_sum_kernel(const Packed a, int32_t size, int32_t blocks)
{
    const int32_t item = (int32_t)blockIdx.x / blocks;
    const int32_t slot = item / a.kv_heads, kvh = item - slot * a.kv_heads;
    const Segment s = segment_of<OWN>(a, slot, 1, false);
    const int64_t begin = (int64_t)s.tile * OWN;
    if (s.none || begin >= s.count)
        return;
    const Walk walk(a, s, OWN, size);
    if (walk.parts == 1) // written as it should be
        return;
    const int64_t lines = (int64_t)a.tokens * a.kv_heads;
    const int32_t quads = a.dim / 4;
    for (int32_t quarter = (int32_t)blockIdx.x - item * blocks; quarter < 4; quarter += blocks) {
        const int32_t half = quarter & 1, which = quarter >> 1;
        const int32_t key0 = (int32_t)begin + half * (OWN / 2), left = s.count - key0, keys = left < OWN / 2 ? left : OWN / 2;
        for (int32_t i0 = (int32_t)threadIdx.x; i0 < keys * quads; i0 += 4 * 256) {
            f32x4 v[4] = {};
            int64_t place[4]; // of the four elements, in [tokens, kv_heads, dim]
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int32_t i = i0 + 256 * n < keys * quads ? i0 + 256 * n : i0, row = i / quads;
                place[n] = (((int64_t)s.first + key0 + row) * a.kv_heads + kvh) * a.dim + 4 * (i - row * quads);
            }
            for (int32_t p = 0; p < walk.parts; ++p) {
                const float *const from = a.partial + (2 * p + which) * lines * a.dim;
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    v[n] += *reinterpret_cast<const f32x4 *>(from + place[n]);
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                if (i0 + 256 * n >= keys * quads)
                    break;
                u32x2 o;
                o[0] = Matrix<IO>::two(v[n][0], v[n][1]);
                o[1] = Matrix<IO>::two(v[n][2], v[n][3]);
                *reinterpret_cast<u32x2 *>((which ? a.dv : a.dk) + place[n] * 2) = o;
            }
        }
    }
}

// dQ of 32 rows a wavefront.
template <class SH, int PARTS, bool FINE> __global__ __launch_bounds__(256, 2) void causal_queries_kernel(const Packed a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, ND = DP / 32, NS = DP / 16, KT = 64, KEYS = KT / PARTS, kOwn = 32 * SH::kWaves / PARTS;
    static_assert(PARTS == 1 || (size_t)2 * (DP / 8) * 64 * 16 <= SH::kRowLds, ""); // what the wavefronts join
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5, group = (uint32_t)a.group;
    const int32_t turn = (int32_t)blockIdx.x / a.kv_heads, kvh = (int32_t)blockIdx.x - turn * a.kv_heads;
    const Segment s = segment_of<kOwn>(a, turn, a.group, true);
    const int own = wave / PARTS, shared = wave % PARTS;
    const int32_t all = s.count * a.group;
    const int64_t begin = (int64_t)s.tile * kOwn;
    if (begin >= all)
        return;
    const uint32_t row0 = (uint32_t)begin + (uint32_t)own * 32u, row = row0 + col;
    const bool there = (int32_t)row < all, works = (int32_t)row0 < all && !s.none;
    // keys: of the workgroup up to its last row's, of the wavefront all below `from`, none from `to` on
    const int32_t last = (int32_t)((uint32_t)begin + kOwn - 1 < (uint32_t)all ? (uint32_t)begin + kOwn - 1 : (uint32_t)all - 1) / a.group;
    const int32_t end = s.none ? 0 : last + 1;
    const int32_t from = (int32_t)(row0 / group) + 1, to = (int32_t)((row0 + 31u) / group) + 1, query = (int32_t)(row / group);
    const int32_t tiles = (end + KT - 1) / KT;
    const LastTwiceLoads<DP, KT, SH::kWaves> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    RowOperand<DP> row_operand(lane);
    ColumnOperand<DP> column_operand(lane);
    row_operand.move(row_at<DP>((uint32_t)(KEYS * shared)));
    column_operand.move(row_at<DP>((uint32_t)(KEYS * shared)));
    const uint64_t k_base = a.k.at + (uint64_t)((int64_t)s.first * a.k.token + kvh * a.k.head);
    const uint64_t v_base = a.v.at + (uint64_t)((int64_t)s.first * a.v.token + kvh * a.v.head);
    if (a.dim < DP) {
#pragma unroll 1
        for (uint32_t at = 0; at < 2 * SH::kRowStage; at += SH::kRowStage) {
            k_loads.clear(lane, lds0 + at);
            v_loads.clear(lane, lds0 + at + SH::kKeysTile);
        }
    }
    auto issue = [&](int32_t t, uint32_t at) {
        k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, a.k.token, a.dim, end - t * KT, lds0 + at);
        v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, a.v.token, a.dim, end - t * KT, lds0 + at + SH::kKeysTile);
    };
    if (tiles > 0)
        issue(0, 0);
    u32x4 q[NS], o[NS];
    {
        const uint64_t q_at = a.q.at + (uint64_t)((int64_t)s.first * a.q.token + (int64_t)kvh * a.group * a.q.head + row_offset(row, group, a.q.token, a.q.head));
        const uint64_t o_at =
            a.dout.at + (uint64_t)((int64_t)s.first * a.dout.token + (int64_t)kvh * a.group * a.dout.head + row_offset(row, group, a.dout.token, a.dout.head));
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            const uint32_t channel = 16u * st + 8u * h;
            const bool loaded = there && channel < (uint32_t)a.dim;
            q[st] = gload16(loaded ? q_at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            o[st] = gload16(loaded ? o_at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
    }
    const float c = a.c;
    const int64_t place = packed_row(a, s, row);
    float up = 1.0f; // of the row
    float lse = there ? a.lse[(int64_t)kvh * a.rows + place] : __builtin_inff();
    float delta = 0.0f;
    if constexpr (kRowsFirst<IO>) {
        float largest = 0.0f;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                largest = fmaxf(largest, fmaxf(fabsf(MM::first(o[st][j])), fabsf(MM::second(o[st][j]))));
        up = scale_of(__builtin_bit_cast(uint32_t, halves_max(largest)));
        const int32_t base = place_of<kGroup>(s.first, 1, s.index), groups = (end + kGroup - 1) / kGroup;
        uint32_t longest = 0;
        for (int32_t i = lane; i < groups; i += 64) {
            const f32x4 values = reinterpret_cast<const f32x4 *>(a.value_most)[(int64_t)kvh * a.value_tiles + base + i];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                longest = kGroup * i + 32 * j < s.count ? greater(longest, values[j]) : longest; // (the others are nobody's)
        }
        delta = there && !s.none ? a.row_delta[(int64_t)kvh * a.rows + place] : 0.0f;
        up = lowered(up, __builtin_bit_cast(float, most_of_lanes(longest)), fabsf(delta), a.dim);
        delta *= up;
    } else {
        // for the keys' kernel too
        const uint64_t at = a.forward_out + (uint64_t)packed_at(a, s, kvh, row), rest = reinterpret_cast<uint64_t>(a.rest) + (uint64_t)packed_at(a, s, kvh, row);
        u32x4 y[NS], z[NS];
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            const uint32_t channel = 16u * st + 8u * h;
            const bool loaded = there && channel < (uint32_t)a.dim;
            y[st] = gload16(loaded ? at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            z[st] = gload16(loaded && a.rest ? rest + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                delta += MM::first(o[st][j]) * (MM::first(y[st][j]) + MM::first(z[st][j])) + MM::second(o[st][j]) * (MM::second(y[st][j]) + MM::second(z[st][j]));
        delta = halves_sum(delta);
        if (h == 0 && there && shared == 0)
            a.row_delta[(int64_t)kvh * a.rows + place] = delta;
    }
    f32x16 dq[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        dq[d] = f32x16{};

    arrived(q);
    arrived(o);
    arrived(lse);
    arrived(delta);
    uint32_t at = 0;
#pragma unroll 1
    for (int32_t t = 0; t < tiles; ++t) {
        wait_loads<0>();
        barrier();
        if (t + 1 < tiles)
            issue(t + 1, at ^ SH::kRowStage);
        const auto rows = row_operand.moved(lds0 + at);
        const auto columns = column_operand.moved(lds0 + at);
        at ^= SH::kRowStage;
        const int32_t key0 = t * KT + KEYS * shared; // the wavefront's first
        if (!works || key0 >= to)
            continue;
        const bool crossed = key0 + KEYS > from;
#pragma unroll
        for (int kb = 0; kb < KEYS / 32; ++kb) {
            fence_schedule(); // (the two halves mixed take more registers than there are)
            f32x16 x = {}, d = {};
            {
                constexpr int kAhead = 2;
                u32x4 y[kAhead], z[kAhead];
                auto read = [&](int st) {
                    y[st % kAhead] = RowOperand<DP>::read(rows, kb, st);
                    z[st % kAhead] = RowOperand<DP>::read(rows, kb, st, SH::kKeysTile);
                };
#pragma unroll
                for (int st = 0; st < kAhead; ++st)
                    read(st);
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    x = MM::multiply(y[st % kAhead], q[st], x);
                    d = MM::multiply(z[st % kAhead], o[st], d);
                    if (st + kAhead < NS)
                        read(st + kAhead);
                    fence_schedule();
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse)) * fmaf(d[i], up, -delta);
            if (crossed) {
                const int32_t seen = query - key0 - 32 * kb - 4 * (int32_t)h;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = 8 * (i / 4) + i % 4 <= seen ? x[i] : 0.0f;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                u32x4 w, left;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = MM::two(x[8 * half + 2 * j], x[8 * half + 2 * j + 1]);
                    if constexpr (FINE)
                        left[j] = rest_of<MM>(w[j], x[8 * half + 2 * j], x[8 * half + 2 * j + 1]);
                }
#pragma unroll
                for (int n = 0; n < ND; ++n) {
                    const u32x4 column = ColumnOperand<DP>::read(columns, kb, half, n);
                    dq[n] = MM::multiply(column, w, dq[n]);
                    if constexpr (FINE)
                        dq[n] = MM::multiply(column, left, dq[n]);
                }
            }
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 8, 0);
#pragma unroll
            for (int n = 0; n < 2 * ND - 4; ++n) {
                __builtin_amdgcn_sched_group_barrier(kProducts, FINE ? 2 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kProducts, FINE ? 8 : 4, 0);
        }
    }

    if constexpr (PARTS > 1) // the first adds what the second has
        if (!add_second<ND>(smem, own, shared, lane, [&](int n) -> f32x16 & { return dq[n]; }))
            return;
    if (!there)
        return;
    const float by = a.scale / up;
    char *const out = a.out + packed_at(a, s, kvh, row);
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int channel = 32 * n + 8 * g + 4 * (int)h;
            if (channel >= a.dim)
                continue;
            u32x2 w;
            w[0] = MM::two(dq[n][4 * g] * by, dq[n][4 * g + 1] * by);
            w[1] = MM::two(dq[n][4 * g + 2] * by, dq[n][4 * g + 3] * by);
            *reinterpret_cast<u32x2 *>(out + channel * 2) = w;
        }
}

// ------------------------------------------------------------------------------------------------ host

typedef void (*Kernel)(Packed);
struct CausalBack {
    Kernel rows, keys, queries;
    void (*sum)(Packed, int32_t, int32_t);
    int size, own; // of the keys' kernel: rows of a stage, keys of a workgroup
    int at_once;   // workgroups of it that the device holds
    size_t keys_lds, queries_lds;
    int64_t keys_slots, queries_slots;
};
template <class KEYS, int PARTS> static CausalBack variant(const Packed &a)
{
    using IO = typename KEYS::IO;
    using QUERIES = BackShape<IO, KEYS::DP, 64, false, 2>;
    CausalBack v = {causal_rows_kernel<IO>, causal_keys_kernel<KEYS>, causal_queries_kernel<QUERIES, PARTS, KEYS::FINE>, causal_sum_kernel<IO, KEYS::kOwn>, KEYS::ROWS, KEYS::kOwn,
                    256 * KEYS::PER, KEYS::kKeyLds, QUERIES::kRowLds, slots_of<KEYS::kOwn>(a, 1), slots_of<128 / PARTS>(a, a.group)};
    return v;
}
template <typename IO, bool FINE> static CausalBack pick(const Packed &a)
{
    // (as for rows.  us of forward and backward without and with, twelve heads of 64: 24 sequences of 60 to 1,000 tokens 92.7 / 78.2, eight
    // of 240 to 4,000 256 / 226, one of 4,096 189 / 179, 60 of 18 to 300 71.8 / 67.5, 30 of 60 to 1,000 103.4 / 97.9; 40 136 / 143, sixteen
    // of 240 to 4,000 462 / 485)
    const bool rows = few_rows(a), keys = slots_of<128>(a, 1) * a.kv_heads <= 1408;
    auto with = [&](auto one, auto two) {
        using ONE = decltype(one);
        using TWO = decltype(two);
        return keys ? rows ? variant<TWO, 2>(a) : variant<TWO, 1>(a) : rows ? variant<ONE, 2>(a) : variant<ONE, 1>(a);
    };
    if (a.dim <= 32)
        return with(CausalBackShape<IO, 32, 64, false, 2, 1, FINE>{}, CausalBackShape<IO, 32, 64, false, 2, 2, FINE>{});
    if (a.dim <= 64)
        return with(CausalBackShape<IO, 64, 32, true, 3, 1, FINE>{}, CausalBackShape<IO, 64, 64, true, 3, 2, FINE>{});
    if (a.dim <= 96)
        return with(CausalBackShape<IO, 96, 64, false, 2, 1, FINE>{}, CausalBackShape<IO, 96, 64, false, 2, 1, FINE>{});
    return with(CausalBackShape<IO, 128, 32, true, 2, 1, FINE>{}, CausalBackShape<IO, 128, 32, true, 2, 1, FINE>{});
}

// S' in two parts where sequences are short: longer ones average more, and pay more.  us of forward and backward with one part and with
// two: 32 sequences of up to 100 tokens, 32 heads of 128 on eight 68.3 / 70.4, ten of up to 100, twelve of 64 66 / 66, sixteen of 90 to
// 1,500 110.5 / 116, one of 1,000, 32 of 128 on eight 104.5 / 112, 4,001 and 2,852, 16 on four 517 / 591.  The host knows the average alone,
// and empty sequences lower it: a short sequence that is packed with a long one has one part, and a long one behind many empty ones two.
template <typename IO> static CausalBack pick(const Packed &a)
{
    return (int64_t)a.tokens < 128 * (int64_t)a.sequences ? pick<IO, true>(a) : pick<IO, false>(a);
}

struct CausalPlan {
    CausalBack v;
    Packed a;
    size_t row_most, value_most, stats, partial; // elements of the workspace: in front of the largest of the rows, of the values' lengths and of the parts; of the parts
};

static CausalPlan plan(const Packed &given, grkan_dtype_t io)
{
    CausalPlan p;
    p.v = io == GRKAN_BF16 ? pick<__bf16>(given) : pick<_Float16>(given);
    Packed &a = p.a;
    a = given;
    a.row_tiles = (int32_t)slots_of<kRowTile>(a, a.group);
    a.value_tiles = (int32_t)slots_of<kGroup>(a, 1);
    a.key_tiles = (int32_t)p.v.keys_slots;
    a.slots = (int32_t)p.v.queries_slots;
    // Slabs, of 1.4 times what each workgroup has to do on the average, if the sequences were all of one length, which the host does not
    // know (empty ones count: 4,001 and 2,852 tokens with 510 empty sequences behind 926 us forward and backward, in the place of 506): so
    // many that the device holds them all at once.  Where a sequence is longer its parts are the more, and then the longer (Walk). There is
    // a workgroup for each part that there may be, and most are not there: not so many that these take time themselves, 1.5 us each, nor
    // more than a GB of sums.  us of the keys' kernel + the sum, with slabs of 1.4, 1.0 and 0.5 of the average: 4,001 and 2,852 tokens, 16
    // heads of 128 on four 261 + 13, 304 + 16, 289 + 22; one of 4,096, twelve of 64 80 + 10, 87 + 12, 83 + 14.  1,024 and 512 rows at
    // least: one of 1,000, 32 heads of 128 on eight 67 + 8, 46 + 11; of 577, twelve of 64 15.8 + 0, 14.9 + 3.9.
    const int64_t each = a.sequences > 0 ? ((int64_t)a.tokens + a.sequences - 1) / a.sequences : 0;
    const int64_t walk = (each * a.group + p.v.size - 1) / p.v.size, longest = (a.rows + p.v.size - 1) / p.v.size; // tiles of rows: of a first key, at most
    const int64_t share = (int64_t)a.kv_heads * ((a.tokens + p.v.own - 1) / p.v.own) * walk / 2 / p.v.at_once;
    const int64_t slab = std::max<int64_t>(share * 7 / 5, (a.dim <= 64 ? 1024 : 512) / p.v.size), wanted = (longest + slab - 1) / slab;
    const int64_t turns = 1 + 2 * (int64_t)p.v.at_once / ((int64_t)a.key_tiles * a.kv_heads);
    const int64_t part = 2 * (int64_t)a.tokens * a.kv_heads * a.dim, held = ((int64_t)1 << 28) / (part > 0 ? part : 1);
    a.slab = (int32_t)slab;
    a.parts = (int32_t)std::max<int64_t>(1, std::min({wanted, turns, held, (int64_t)16}));
    p.row_most = ((size_t)a.kv_heads * (size_t)a.rows + 3) & ~(size_t)3;
    p.value_most = p.row_most + ((2 * (size_t)a.kv_heads * (size_t)a.row_tiles + 3) & ~(size_t)3);
    p.stats = p.value_most + 4 * (size_t)a.kv_heads * (size_t)a.value_tiles;
    p.partial = a.parts > 1 ? (size_t)a.parts * (size_t)part : 0;
    return p;
}

} // namespace attention
} // namespace grkan

using namespace grkan;

extern "C" size_t grkan_causal_attention_bwd_workspace_bytes(const grkan_causal_attention_t *at)
{
    attention::Packed a;
    if (attention::fill(at, GRKAN_BF16, &a) != GRKAN_OK)
        return 0;
    const attention::CausalPlan p = attention::plan(a, GRKAN_BF16);
    return (p.stats + p.partial) * sizeof(float);
}

extern "C" grkan_status_t grkan_causal_attention_bwd(const grkan_causal_attention_t *at, const void *out, const void *rest, const float *lse, const void *dout,
                                                     int64_t dout_token_stride, int64_t dout_head_stride, void *dq, void *dk, void *dv, void *workspace,
                                                     size_t workspace_bytes, grkan_dtype_t io, void *hip_stream)
{
    attention::Packed given;
    const grkan_status_t bad = attention::fill(at, io, &given);
    if (bad != GRKAN_OK)
        return bad;
    if (given.tokens == 0)
        return GRKAN_OK;
    if (!out || !lse || !dout || !dq || !dk || !dv)
        return GRKAN_ERR_NULL;
    auto address = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if ((address(out) | address(rest) | address(dout) | address(dq) | address(dk) | address(dv)) % 16 != 0 || address(lse) % 4 != 0 ||
        (dout_token_stride | dout_head_stride) % 8 != 0)
        return GRKAN_ERR_ALIGN;
    if (!attention::in_offsets(dout_token_stride, dout_head_stride, given.group))
        return GRKAN_ERR_UNSUPPORTED;
    attention::CausalPlan p = attention::plan(given, io);
    const size_t need = (p.stats + p.partial) * sizeof(float);
    if (!workspace || workspace_bytes < need || address(workspace) % 16 != 0)
        return GRKAN_ERR_WORKSPACE;
    attention::Packed &a = p.a;
    const int64_t heads = a.kv_heads, rows_grid = heads * a.row_tiles, keys_grid = heads * a.key_tiles * a.parts;
    const int64_t queries_grid = heads * a.slots;
    a.dout = attention::Operand{address(dout), 0, dout_token_stride * 2, dout_head_stride * 2};
    a.lse = const_cast<float *>(lse);
    a.row_delta = static_cast<float *>(workspace);
    a.row_most = a.row_delta + p.row_most;
    a.value_most = a.row_delta + p.value_most;
    a.partial = a.row_delta + p.stats;
    a.dk = static_cast<char *>(dk);
    a.dv = static_cast<char *>(dv);
    a.forward_out = address(out);
    a.rest = static_cast<char *>(const_cast<void *>(rest));
    a.out = static_cast<char *>(dq);
    if (!attention::allow_lds(reinterpret_cast<const void *>(p.v.keys), p.v.keys_lds) ||
        !attention::allow_lds(reinterpret_cast<const void *>(p.v.queries), p.v.queries_lds))
        return GRKAN_ERR_LAUNCH;
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    auto launch = [&](attention::Kernel kernel, int64_t grid, size_t lds) {
        void *args[] = {&a};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)grid), dim3(256), args, lds, stream) == hipSuccess;
    };
    auto keys = [&] {
        if (!launch(p.v.keys, keys_grid, p.v.keys_lds))
            return false;
        if (a.parts == 1)
            return true;
        // four to a tile where the device holds them all (eight on a compute unit; sixteen sequences of 90 to 1,500 tokens, twelve heads of
        // 64: 11.5 us with four, 8.2 with one)
        const int64_t tiles = heads * a.key_tiles;
        int32_t size = p.v.size, blocks = 4 * tiles <= 2048 ? 4 : 1;
        void *args[] = {&a, &size, &blocks};
        return hipLaunchKernel(reinterpret_cast<const void *>(p.v.sum), dim3((unsigned)(tiles * blocks)), dim3(256), args, 0, stream) == hipSuccess;
    };
    // each needs what the other leaves: the lengths of the values, or the rows' statistics
    if (io == GRKAN_F16)
        return launch(p.v.rows, rows_grid, 0) && keys() && launch(p.v.queries, queries_grid, p.v.queries_lds) ? GRKAN_OK : GRKAN_ERR_LAUNCH;
    return launch(p.v.queries, queries_grid, p.v.queries_lds) && keys() ? GRKAN_OK : GRKAN_ERR_LAUNCH;
}
