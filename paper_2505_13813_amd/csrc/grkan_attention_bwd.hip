// Cross attention on gfx950 (MI355X), backward.  With P recomputed from the rows' lse and D = dO V^T:
//
//     dV = P^T dO        S' = P (D - delta), delta = the row's sum of dO O        dQ = scale S' K        dK = scale S'^T Q
//
// Seven products as they stand (the scores and D twice), in two kernels, so that every gradient is summed by whoever owns it: no
// atomics, the same bits each time.  One has keys, walks the rows and keeps dK and dV; the other has rows, walks the keys and
// keeps dQ.  In both, as in the forward pass, the product that is contracted next is left in the registers as the operand of the next.
// delta is made by the queries' kernel, or in front of both by a small one.
//
// Bound by the products and the vector operations between them (two fused multiply-adds, an exponential and a rounding for each score), of which little
// runs at once, and waiting for the next stage: the matrix units are busy for 42 % (keys) and 53 % (queries) of the time with 128 channels, 26 and 30 % with 64, and the
// wavefronts wait for 51, 41, 39 and 34 %.  2 x 4096 queries, 4,001 and 1,808 keys, 16 heads of 128 that read four, float16: keys' kernel 459 - 472 us = 830 - 850
// TFLOP/s, queries' 297 - 307 us = 950 - 985, where a large library product reaches 1,500; rows 15, sums 24.  32 x 256 queries, 785 keys, 12 heads of 64,
// bfloat16: 80 - 84 and 51 - 55.
//
// float16: S' of a small upstream gradient would be below its range.  The products take 2^e S', with e such that the largest |dO| becomes 1/4 to
// 1/2, and the sums are scaled back in float32.  For dQ it is the largest of the row, which
// no other row has a part in: with one e for all, a row 2^-12 as large as the largest was off by 6 % (4,001 keys of 128 channels; 0.03 % so).  For dK, a sum
// over rows, it is the largest of the key head.  |S'| is at most |D| + |delta|, and |D| at most sqrt(dim) max |dO| times the value's length: where that
// passes half of the type's range (values from some 250 on in all of 128 channels), e is lowered, for dK by the key's own value, for dQ by the key
// head's longest one, which the keys' kernel leaves.  (Without that, values of 20,000 and a third of a row's probability made S' infinite.
// 32 x 256 queries, 785 keys, 12 heads of 64 with a mask, float16, forward and backward: 168 us without, 170 so.)
#include <hip/hip_runtime.h>

#include "grkan_attention_back.h"

namespace grkan {
namespace attention {

// float16: delta, and copies of lse, of 64 rows for each workgroup: sixteen lanes a row, eight channels each.  (bfloat16, which is not scaled, needs no launch in
// front: the queries' kernel has the rows of dO in its registers, reads those of O once, and leaves both for the keys' kernel behind it.  32 x 256 queries of
// 12 heads of 64, 785 keys and a mask, forward and all gradients: 158 us in the place of 164.)
template <typename IO> __global__ __launch_bounds__(256) void rows_kernel(const Args a)
{
    using MM = Matrix<IO>;
    __shared__ uint32_t most[4][2];
    const int32_t tiles = a.padded / kRowTile;
    const int32_t bh = (int32_t)blockIdx.x / tiles, tile = (int32_t)blockIdx.x - bh * tiles;
    const int32_t b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    const uint32_t lane16 = threadIdx.x & 15u;
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    const uint64_t out = a.forward_out + 2u * (uint64_t)((int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim);
    const uint64_t dout = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head);
    const uint32_t row0 = (uint32_t)tile * kRowTile + (threadIdx.x >> 4);
    u32x4 o[4], d[4];
    float lse[4], largest = 0.0f, sums = 0.0f;
    // (all loads in front, without a branch: they wait for one another otherwise)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t row = row0 + 16u * k;
        const bool there = (int64_t)row < a.rows, loaded = there && 8u * lane16 < (uint32_t)a.dim;
        const uint64_t zeros = reinterpret_cast<uint64_t>(kZeros);
        o[k] = gload16(loaded ? out + 2u * (uint64_t)row_offset(row, (uint32_t)a.group, heads_dim, a.dim) + 16u * lane16 : zeros, 0);
        d[k] = gload16(loaded ? dout + (uint64_t)row_offset(row, (uint32_t)a.group, a.dout.token, a.dout.head) + 16u * lane16 : zeros, 0);
        const float *const from = there ? a.lse + ((int64_t)bh * a.rows + row) : reinterpret_cast<const float *>(kZeros);
        lse[k] = *from;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t row = row0 + 16u * k;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = MM::first(d[k][j]), y = MM::second(d[k][j]);
            sum += x * MM::first(o[k][j]) + y * MM::second(o[k][j]);
            largest = fmaxf(largest, fmaxf(fabsf(x), fabsf(y)));
        }
#pragma unroll
        for (int s = 8; s > 0; s /= 2)
            sum += __shfl_xor(sum, s);
        sums = fmaxf(sums, fabsf(sum));
        if (lane16 == 0) {
            const int64_t at = (int64_t)bh * a.padded + row;
            a.row_lse[at] = (int64_t)row < a.rows ? lse[k] : __builtin_inff();
            a.row_delta[at] = sum;
        }
    }
    const uint32_t bits[2] = {most_of_lanes(__builtin_bit_cast(uint32_t, largest)), most_of_lanes(__builtin_bit_cast(uint32_t, sums))};
    if ((threadIdx.x & 63) == 0) {
        most[threadIdx.x >> 6][0] = bits[0];
        most[threadIdx.x >> 6][1] = bits[1];
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        uint32_t all = 0;
        for (int w = 0; w < 4; ++w)
            all = most[w][threadIdx.x] > all ? most[w][threadIdx.x] : all;
        a.row_most[2 * ((int64_t)bh * tiles + tile) + threadIdx.x] = __builtin_bit_cast(float, all);
    }
}

// How many workgroups share the walk over the rows of each of `groups` groups of keys, `most` in all: what makes their last round on the device a full
// one, counted in tiles of rows.  A part costs three to begin with, and where there are several, their way to the workspace and back is that of about
// 32 for 512 parts.  (188 groups of 128 keys, 16,384 rows of 128 channels, 512 workgroups at once: 535 us with 2 parts, 465 with 5.)
__host__ __device__ __forceinline__ int32_t parts_of(int64_t groups, int32_t tiles, int32_t at_once, int32_t most)
{
    int32_t best = 1;
    int64_t least = INT64_MAX;
    for (int32_t n = 1; n <= 8; ++n) {
        const int64_t all = groups * n;
        if (n > 1 && (all > most || 4 * n > tiles))
            break;
        const int64_t cost = (all + at_once - 1) / at_once * ((tiles + n - 1) / n + 3) + (n > 1 ? all / 16 : 0);
        if (cost < least) {
            least = cost;
            best = n;
        }
    }
    return best;
}

// dK and dV of 32 keys a wavefront, of a group of 128 a workgroup, from all rows or, where there are few groups (a.splits), from a part of them.
template <class SH> __global__ __launch_bounds__(256, SH::PER) void keys_kernel(const Args a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, ROWS = SH::ROWS, ND = DP / 32, NS = DP / 16;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    const int32_t item = work_item(a);
    if (item >= a.work)
        return;
    const int32_t tiles = (int32_t)((a.rows + ROWS - 1) / ROWS);
    int32_t b, kvh, key_tile, count, t0 = 0, t1 = tiles;
    bool whole = true;
    if (a.splits) {
        Deal deal(a);
        const int32_t parts = parts_of(deal.total, tiles, a.at_once, a.splits), g = item / parts, per = (tiles + parts - 1) / parts;
        if (g >= deal.total)
            return;
        deal.find(a, g);
        b = deal.b;
        count = deal.count;
        kvh = (g - deal.begin) / deal.groups;
        key_tile = g - deal.begin - kvh * deal.groups;
        t0 = (item - g * parts) * per;
        t1 = t0 + per < tiles ? t0 + per : tiles;
        whole = parts == 1;
    } else {
        const int32_t bh = item / a.key_tiles;
        key_tile = item - bh * a.key_tiles;
        b = bh / a.kv_heads;
        kvh = bh - b * a.kv_heads;
        count = keys_of(a, b);
        if ((int64_t)key_tile * SH::kOwn >= count) // no valid key in the workgroup: zeros
            t1 = 0;
    }
    const int32_t bh = b * a.kv_heads + kvh;
    const int64_t key0 = (int64_t)key_tile * SH::kOwn + wave * 32, key = key0 + col; // this wavefront's and this lane's

    // ---- keys and values as second operands: lane l has key l mod 32, channels 16 s + 8 (l / 32) ..
    u32x4 k[NS], v[SH::V_LDS ? 1 : NS];
    const bool valid = key < count && (!a.mask || a.mask[(int64_t)b * a.mask_batch + key * a.mask_key] != 0);
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const uint32_t channel = 16u * s + 8u * h;
        const bool there = valid && channel < (uint32_t)a.dim;
        k[s] = gload16(there ? k_base + (uint64_t)key * (uint64_t)a.k.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        if constexpr (!SH::V_LDS)
            v[s] = gload16(there ? v_base + (uint64_t)key * (uint64_t)a.v.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
    }

    f32x16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        dk[d] = f32x16{};
        dv[d] = f32x16{};
    }

    const RowOperand<DP> row_operand(lane);
    const ColumnOperand<DP> column_operand(lane);
    const uint64_t q_base = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head);
    const uint64_t d_base = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head);
    const RowLoads<DP, ROWS, SH::kWaves> q_loads(wave, lane, a.q, q_base, a.even_q && ROWS % a.group == 0, a),
        d_loads(wave, lane, a.dout, d_base, a.even_dout && ROWS % a.group == 0, a);
    const bool works = key0 < count; // (a wavefront without keys loads for the others)
    const float c = a.c;
    float up = 1.0f; // of the key
    if constexpr (kRowsFirst<IO>) {
        u32x4 value[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool there = valid && channel < (uint32_t)a.dim;
            value[s] = gload16(there ? v_base + (uint64_t)key * (uint64_t)a.v.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
        const int32_t row_tiles = a.padded / kRowTile;
        uint32_t largest = 0, sums = 0;
        for (int32_t i = lane; i < row_tiles; i += 64) {
            const f32x2 both = reinterpret_cast<const f32x2 *>(a.row_most)[(int64_t)bh * row_tiles + i];
            largest = greater(largest, both[0]);
            sums = greater(sums, both[1]);
        }
        float length2 = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                length2 += MM::first(value[s][j]) * MM::first(value[s][j]) + MM::second(value[s][j]) * MM::second(value[s][j]);
        length2 = halves_sum(length2);
        up = lowered(scale_of(most_of_lanes(largest)), length2, __builtin_bit_cast(float, most_of_lanes(sums)), a.dim);
        const uint32_t longest = most_of_lanes(__builtin_bit_cast(uint32_t, length2) & 0x7fffffffu);
        if (lane == 0) // (the same by all that share the group)
            a.value_most[((int64_t)bh * a.key_tiles + key_tile) * SH::kWaves + wave] = __builtin_bit_cast(float, longest);
    }

    auto issue = [&](int32_t t, uint32_t stage) {
        const uint32_t row0 = (uint32_t)t * ROWS;
        q_loads.issue(a.q, t, a.rows, a, stage);
        d_loads.issue(a.dout, t, a.rows, a, stage + SH::kRowsTile);
        // (the rows' statistics are padded to whole tiles of 64)
        if (wave < 2 && lane < ROWS) {
            const float *const from = (wave ? a.row_delta : a.row_lse) + (int64_t)bh * a.padded + row0;
            load_words_to_lds(uniform_u64(reinterpret_cast<uint64_t>(from)), (uint32_t)lane * 4u, stage + 2 * SH::kRowsTile + (uint32_t)wave * ROWS * 4u);
        }
    };

    const uint32_t stages = lds0 + (SH::V_LDS ? 2 * SH::kKeysTile : 0u);
    uint32_t at = SH::kKeyStage;
    if constexpr (SH::V_LDS) {
        if (t0 < t1) {
            const TileLoads<DP, 64, SH::kWaves> v_loads(wave, lane, a.v.token, a.dim);
#pragma unroll 1
            for (int part = 0; part < 2; ++part) {
                const int64_t first = (int64_t)key_tile * SH::kOwn + 64 * part, mine = first + lane;
                const bool there = mine < count && (!a.mask || a.mask[(int64_t)b * a.mask_batch + mine * a.mask_key] != 0);
                v_loads.issue(v_base + (uint64_t)first * (uint64_t)a.v.token, a.v.token, __ballot(there), false, lds0 + (uint32_t)part * SH::kKeysTile);
            }
        }
    }
    arrived(k);
    if constexpr (!SH::V_LDS)
        arrived(v);
    const auto v_rows = row_operand.moved(lds0 + (uint32_t)wave * row_at<DP>(32u));
#pragma unroll 1
    for (int32_t t = t0 - 1; t < t1; ++t) {
        if (t >= t0) {
            wait_loads<0>();
            barrier();
        }
        if (t + 1 < t1)
            issue(t + 1, stages + (at ^ SH::kKeyStage));
        const uint32_t stage = stages + at;
        at ^= SH::kKeyStage;
        if (t < t0 || !works)
            continue;
        const auto rows = row_operand.moved(stage);
        const auto columns = column_operand.moved(stage);
        uint32_t stats = stage + 2 * SH::kRowsTile + 16u * h;
#pragma unroll
        for (int rb = 0; rb < ROWS / 32; ++rb) {
            f32x16 p = {}, d = {};
#pragma unroll
            for (int st = 0; st < NS; ++st)
                p = MM::multiply(RowOperand<DP>::read(rows, rb, st), k[st], p);
            u32x4 w[2];
#pragma unroll
            for (int quad = 0; quad < 4; ++quad) {
                const f32x4 lse = __builtin_bit_cast(f32x4, lds_read16(stats + (32u * rb + 8u * quad) * 4u));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    p[4 * quad + j] = __builtin_amdgcn_exp2f(fmaf(p[4 * quad + j], c, -lse[j]));
                w[quad / 2][2 * (quad % 2)] = MM::two(p[4 * quad], p[4 * quad + 1]);
                w[quad / 2][2 * (quad % 2) + 1] = MM::two(p[4 * quad + 2], p[4 * quad + 3]);
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                u32x4 value;
                if constexpr (SH::V_LDS)
                    value = RowOperand<DP>::read(v_rows, 0, st);
                else
                    value = v[st];
                d = MM::multiply(RowOperand<DP>::read(rows, rb, st, SH::kRowsTile), value, d);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int part = 0; part < ND; ++part)
                    dv[part] = MM::multiply(ColumnOperand<DP>::read(columns, rb, half, part, SH::kRowsTile), w[half], dv[part]);
#pragma unroll
            for (int quad = 0; quad < 4; ++quad) {
                const f32x4 delta = __builtin_bit_cast(f32x4, lds_read16(stats + (ROWS + 32u * rb + 8u * quad) * 4u));
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = p[4 * quad + j] * fmaf(d[4 * quad + j], up, -delta[j] * up);
                w[quad / 2][2 * (quad % 2)] = MM::two(y[0], y[1]);
                w[quad / 2][2 * (quad % 2) + 1] = MM::two(y[2], y[3]);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int part = 0; part < ND; ++part)
                    dk[part] = MM::multiply(ColumnOperand<DP>::read(columns, rb, half, part), w[half], dk[part]);
        }
    }

    if (key >= a.keys)
        return;
    const float by = a.scale / up;
    const int64_t line = ((int64_t)b * a.keys + key) * a.kv_heads + kvh;
    float *const to = a.partial + ((int64_t)item * 2 * kGroup + (wave * 32 + (int)col)) * a.dim;
#pragma unroll
    for (int part = 0; part < ND; ++part)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int channel = 32 * part + 8 * g + 4 * (int)h;
            if (channel >= a.dim)
                continue;
            f32x4 x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = valid ? dk[part][4 * g + j] * by : 0.0f;
                y[j] = valid ? dv[part][4 * g + j] : 0.0f;
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
                *reinterpret_cast<f32x4 *>(to + kGroup * a.dim + channel) = y;
            }
        }
}

// The sum of the parts of a group of keys, and zeros for a group without keys: block (quarter, dK or dV, group, key head), four elements a lane and pass.
template <typename IO> __global__ __launch_bounds__(256) void sum_keys_kernel(const Args a, int32_t row_tiles)
{
    const int32_t quarter = (int32_t)blockIdx.x & 3, which = (int32_t)blockIdx.x >> 2 & 1, item = (int32_t)blockIdx.x >> 3;
    const int32_t bh = item / a.key_tiles, key_tile = item - bh * a.key_tiles;
    const int32_t b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    Deal deal(a);
    deal.find(a, 0, b);
    int32_t parts = 0;
    if (key_tile < deal.groups) {
        parts = parts_of(deal.total, row_tiles, a.at_once, a.splits);
        if (parts == 1) // written as it should be
            return;
    }
    const int64_t first = (int64_t)(deal.begin + kvh * deal.groups + key_tile) * parts;
    const int32_t quads = a.dim / 4, keys = kGroup / 4, key0 = quarter * keys;
    for (int32_t i = (int32_t)threadIdx.x; i < keys * quads; i += 256) {
        const int32_t row = i / quads, key = key_tile * kGroup + key0 + row;
        if (key >= a.keys)
            break;
        const float *const from = a.partial + ((first * 2 + which) * kGroup + key0) * a.dim + 4 * i;
        f32x4 v = {};
        for (int32_t n = 0; n < parts; ++n)
            v += *reinterpret_cast<const f32x4 *>(from + (int64_t)n * 2 * kGroup * a.dim);
        u32x2 o;
        o[0] = Matrix<IO>::two(v[0], v[1]);
        o[1] = Matrix<IO>::two(v[2], v[3]);
        const int64_t line = ((int64_t)b * a.keys + key) * a.kv_heads + kvh;
        *reinterpret_cast<u32x2 *>((which ? a.dv : a.dk) + (line * a.dim + 4 * (i - row * quads)) * 2) = o;
    }
}

// dQ of 32 rows a wavefront.
template <class SH> __global__ __launch_bounds__(256, 2) void queries_kernel(const Args a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, ND = DP / 32, NS = DP / 16, KT = 64;
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

    const uint32_t row0 = (uint32_t)row_tile * SH::kOwn + (uint32_t)wave * 32u, row = row0 + col;
    const bool there = (int64_t)row < a.rows, works = (int64_t)row0 < a.rows;
    u32x4 q[NS], o[NS];
    {
        const uint64_t q_at = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head +
                                                  row_offset(row, (uint32_t)a.group, a.q.token, a.q.head));
        const uint64_t o_at = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head +
                                                     row_offset(row, (uint32_t)a.group, a.dout.token, a.dout.head));
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool loaded = there && channel < (uint32_t)a.dim;
            q[s] = gload16(loaded ? q_at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            o[s] = gload16(loaded ? o_at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
    }
    const float c = a.c;
    float up = 1.0f; // of the row
    if constexpr (kRowsFirst<IO>) {
        float largest = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                largest = fmaxf(largest, fmaxf(fabsf(MM::first(o[s][j])), fabsf(MM::second(o[s][j]))));
        up = scale_of(__builtin_bit_cast(uint32_t, halves_max(largest)));
        const int32_t groups = Deal::groups_of(keys_of(a, b));
        uint32_t longest = 0;
        for (int32_t i = lane; i < groups; i += 64) {
            const f32x4 values = reinterpret_cast<const f32x4 *>(a.value_most)[(int64_t)bh * a.key_tiles + i];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                longest = greater(longest, values[j]);
        }
        up = lowered(up, __builtin_bit_cast(float, most_of_lanes(longest)), there ? fabsf(a.row_delta[(int64_t)bh * a.padded + row]) : 0.0f, a.dim);
    }
    float lse = there ? a.lse[(int64_t)bh * a.rows + row] : __builtin_inff();
    float delta = 0.0f;
    if constexpr (kRowsFirst<IO>) {
        delta = there ? a.row_delta[(int64_t)bh * a.padded + row] * up : 0.0f;
    } else {
        // the rows' statistics, for the keys' kernel too
        const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
        const uint64_t at = a.forward_out + 2u * (uint64_t)((int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim +
                                                            row_offset(row, (uint32_t)a.group, heads_dim, a.dim));
        u32x4 y[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            y[s] = gload16(there && channel < (uint32_t)a.dim ? at + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                delta += MM::first(o[s][j]) * MM::first(y[s][j]) + MM::second(o[s][j]) * MM::second(y[s][j]);
        delta = halves_sum(delta);
        if (split == 0 && h == 0 && row < (uint32_t)a.padded) {
            a.row_lse[(int64_t)bh * a.padded + row] = lse;
            a.row_delta[(int64_t)bh * a.padded + row] = delta;
        }
    }
    f32x16 dq[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        dq[d] = f32x16{};

    const int32_t count = keys_of(a, b), tiles = (count + KT - 1) / KT;
    int32_t t0 = split * a.tiles_per_split, t1 = t0 + a.tiles_per_split;
    t1 = t1 < tiles ? t1 : tiles;
    const TileLoads<DP, KT, SH::kWaves> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    const RowOperand<DP> row_operand(lane);
    const ColumnOperand<DP> column_operand(lane);
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
    ValidKeys valid(a, b, count, t1);
    arrived(q);
    arrived(o);
    arrived(lse);
    arrived(delta);
    uint32_t at = SH::kRowStage;
    uint64_t word = 0;
#pragma unroll 1
    for (int32_t t = t0 - 1; t < t1; ++t) {
        const uint64_t next = t + 1 < t1 ? valid.word(t + 1) : 0, now = word;
        if (t >= t0) {
            wait_loads<0>();
            barrier();
        }
        if (t + 1 < t1) {
            const bool whole = next == ~(uint64_t)0 && a.dim == DP;
            const uint32_t to = lds0 + (at ^ SH::kRowStage);
            k_loads.issue(k_base + (uint64_t)(t + 1) * KT * (uint64_t)a.k.token, a.k.token, next, whole, to);
            v_loads.issue(v_base + (uint64_t)(t + 1) * KT * (uint64_t)a.v.token, a.v.token, next, whole, to + SH::kKeysTile);
            if (next != ~(uint64_t)0 && wave == 0)
                write_cover(lds0 + SH::kCover + (at ? 0u : KT * 4u), next, lane);
        }
        const uint32_t cover = lds0 + SH::kCover + (at ? KT * 4u : 0u);
        const auto rows = row_operand.moved(lds0 + at);
        const auto columns = column_operand.moved(lds0 + at);
        at ^= SH::kRowStage;
        word = next;
        if (t < t0 || !works || now == 0) // (queries and dO may be NaN where no key is valid)
            continue;
#pragma unroll
        for (int kb = 0; kb < KT / 32; ++kb) {
            fence_schedule(); // (the two halves mixed take more registers than there are)
            f32x16 s, d = {};
            if (now != ~(uint64_t)0) {
                s = read_cover(cover, kb, h);
#pragma unroll
                for (int st = 0; st < NS; ++st)
                    s = MM::multiply(RowOperand<DP>::read(rows, kb, st), q[st], s);
            } else {
                s = f32x16{};
#pragma unroll
                for (int st = 0; st < NS; ++st)
                    s = MM::multiply(RowOperand<DP>::read(rows, kb, st), q[st], s);
            }
#pragma unroll
            for (int st = 0; st < NS; ++st)
                d = MM::multiply(RowOperand<DP>::read(rows, kb, st, SH::kKeysTile), o[st], d);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse)) * fmaf(d[i], up, -delta);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = MM::two(s[8 * half + 2 * j], s[8 * half + 2 * j + 1]);
#pragma unroll
                for (int part = 0; part < ND; ++part)
                    dq[part] = MM::multiply(ColumnOperand<DP>::read(columns, kb, half, part), w, dq[part]);
            }
        }
    }

    if (!there)
        return;
    const float by = a.scale / up;
    const int64_t heads = (int64_t)a.kv_heads * a.group, all = (int64_t)a.batch * a.kv_heads * a.rows;
    const int64_t line = (int64_t)b * (a.rows / a.group) * heads + (int64_t)kvh * a.group + row_offset(row, (uint32_t)a.group, heads, 1);
#pragma unroll
    for (int part = 0; part < ND; ++part)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int channel = 32 * part + 8 * g + 4 * (int)h;
            if (channel >= a.dim)
                continue;
            f32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = dq[part][4 * g + j] * by;
            if (a.splits == 1) {
                u32x2 w;
                w[0] = MM::two(x[0], x[1]);
                w[1] = MM::two(x[2], x[3]);
                *reinterpret_cast<u32x2 *>(a.out + (line * a.dim + channel) * 2) = w;
            } else {
                *reinterpret_cast<f32x4 *>(a.partial + ((int64_t)split * all + line) * a.dim + channel) = x;
            }
        }
}

// The sum of the splits' parts, eight elements a lane.
template <typename IO> __global__ __launch_bounds__(256) void sum_kernel(const float *partial, int32_t splits, int64_t elements, char *out)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= elements)
        return;
    float v[8] = {};
    for (int32_t s = 0; s < splits; ++s) {
        const f32x4 *const from = reinterpret_cast<const f32x4 *>(partial + s * elements + i);
        const f32x4 x = from[0], y = from[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] += x[j];
            v[4 + j] += y[j];
        }
    }
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = Matrix<IO>::two(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<u32x4 *>(out + i * 2) = w;
}

// ------------------------------------------------------------------------------------------------ host

typedef void (*Kernel)(Args);
struct BackVariant {
    Kernel keys, queries;
    int own, rows; // keys or rows of a workgroup; rows of a stage of the keys' kernel
    int at_once;   // workgroups of the keys' kernel that the device holds
    size_t keys_lds, queries_lds;
};
template <class SH> static BackVariant back_variant()
{
    return BackVariant{keys_kernel<SH>, queries_kernel<SH>, SH::kOwn, SH::ROWS, 256 * SH::PER, SH::kKeyLds, SH::kRowLds};
}
template <typename IO> static BackVariant pick(int32_t dim)
{
    if (dim <= 32)
        return back_variant<BackShape<IO, 32, 64, false, 2>>();
    if (dim <= 64)
        return back_variant<BackShape<IO, 64, 32, true, 3>>();
    if (dim <= 96)
        return back_variant<BackShape<IO, 96, 64, false, 2>>();
    return back_variant<BackShape<IO, 128, 32, true, 2>>();
}

struct BackPlan {
    BackVariant v;
    Args keys, queries;
    size_t value_most, stats, partial; // elements of the workspace: up to the values' lengths, up to the parts, of the parts
};

static BackPlan back_plan(const Args &a, grkan_dtype_t io)
{
    BackPlan p;
    p.v = io == GRKAN_BF16 ? pick<__bf16>(a.dim) : pick<_Float16>(a.dim);
    p.keys = p.queries = a;
    const int64_t heads = (int64_t)a.batch * a.kv_heads;
    const int32_t padded = (int32_t)((a.rows + kRowTile - 1) / kRowTile) * kRowTile;
    p.keys.padded = p.queries.padded = padded;
    p.keys.key_tiles = p.queries.key_tiles = (int32_t)((a.keys + p.v.own - 1) / p.v.own);
    p.queries.row_tiles = (int32_t)((a.rows + p.v.own - 1) / p.v.own);
    // Groups of keys that do not fill the device: their walks are shared.  How many of the groups have keys, and so how many share one, the kernel
    // knows, or the host where there are no lengths.
    const int64_t groups = heads * p.keys.key_tiles;
    const int32_t tiles = (int32_t)((a.rows + p.v.rows - 1) / p.v.rows), most = 2 * p.v.at_once;
    p.keys.at_once = p.v.at_once;
    p.keys.splits = 0;
    if (groups > 0 && groups <= p.v.at_once && tiles >= 8) {
        if (a.lengths)
            p.keys.splits = 8 * groups < most ? (int32_t)(8 * groups) : most;
        else if (const int32_t parts = parts_of(groups, tiles, p.v.at_once, most); parts > 1)
            p.keys.splits = (int32_t)groups * parts;
    }
    const int64_t row_work = heads * p.queries.row_tiles, key_tiles = (a.keys + kRowTile - 1) / kRowTile;
    const int64_t splits = splits_of(row_work, key_tiles, a.rows < p.v.own ? a.rows : p.v.own, a.dim, a.dim <= 64 ? 3 : 2, 1.6);
    const int64_t per = (key_tiles + splits - 1) / splits;
    p.queries.tiles_per_split = (int32_t)(per > 1 ? per : 1);
    p.queries.splits = (int32_t)((key_tiles + p.queries.tiles_per_split - 1) / p.queries.tiles_per_split);
    if (p.queries.splits < 1)
        p.queries.splits = 1;
    static_assert(kGroup == 4 * 32, ""); // (a group's lengths are read at once)
    p.value_most = (2 * (size_t)heads * (size_t)padded + 2 * (size_t)heads * (size_t)(padded / kRowTile) + 3) & ~(size_t)3;
    p.stats = p.value_most + 4 * (size_t)heads * (size_t)p.keys.key_tiles;
    // (one after the other: they share the memory)
    const size_t of_keys = 2 * (size_t)p.keys.splits * kGroup * (size_t)a.dim;
    const size_t of_rows = p.queries.splits > 1 ? (size_t)p.queries.splits * (size_t)heads * (size_t)a.rows * (size_t)a.dim : 0;
    p.partial = of_keys > of_rows ? of_keys : of_rows;
    return p;
}

size_t backward_bytes(const Args &a)
{
    const BackPlan p = back_plan(a, GRKAN_BF16);
    return (p.stats + p.partial) * sizeof(float);
}

template <typename IO> static grkan_status_t backward(const BackPlan &p, hipStream_t stream)
{
    const int64_t heads = (int64_t)p.keys.batch * p.keys.kv_heads;
    const int64_t rows_grid = heads * (p.keys.padded / kRowTile);
    Args k = p.keys, q = p.queries;
    const int64_t groups = heads * k.key_tiles, key_work = k.splits ? k.splits : groups, row_work = heads * q.row_tiles * q.splits;
    const int64_t row_elements = heads * k.rows * k.dim, row_blocks = (row_elements / 8 + 255) / 256;
    if (rows_grid > kMostBlocks || key_work > kMostBlocks || row_work > kMostBlocks || (q.splits > 1 && row_blocks > kMostBlocks))
        return GRKAN_ERR_UNSUPPORTED;
    const int64_t row_grid = row_work > 0 ? spread(q, row_work, (int64_t)q.row_tiles * q.splits) : 0;
    const int64_t key_grid = key_work > 0 ? spread(k, key_work, k.splits ? key_work : k.key_tiles) : 0;
    if (row_grid > kMostBlocks || key_grid > kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    if (!allow_lds(reinterpret_cast<const void *>(p.v.keys), p.v.keys_lds) || !allow_lds(reinterpret_cast<const void *>(p.v.queries), p.v.queries_lds))
        return GRKAN_ERR_LAUNCH;
    if constexpr (kRowsFirst<IO>) {
        if (rows_grid > 0)
            rows_kernel<IO><<<dim3((unsigned)rows_grid), 256, 0, stream>>>(k);
    }
    auto queries = [&] {
        if (row_work == 0)
            return true;
        void *args[] = {&q};
        if (hipLaunchKernel(reinterpret_cast<const void *>(p.v.queries), dim3((unsigned)row_grid), dim3(256), args, p.v.queries_lds, stream) != hipSuccess)
            return false;
        if (q.splits > 1)
            sum_kernel<IO><<<dim3((unsigned)row_blocks), 256, 0, stream>>>(q.partial, q.splits, row_elements, q.out);
        return true;
    };
    auto keys = [&] {
        if (key_work == 0)
            return true;
        void *args[] = {&k};
        if (hipLaunchKernel(reinterpret_cast<const void *>(p.v.keys), dim3((unsigned)key_grid), dim3(256), args, p.v.keys_lds, stream) != hipSuccess)
            return false;
        if (k.splits)
            sum_keys_kernel<IO><<<dim3((unsigned)(8 * groups)), 256, 0, stream>>>(k, (int32_t)((k.rows + p.v.rows - 1) / p.v.rows));
        return true;
    };
    // each needs what the other leaves: the lengths of the values, or the rows' statistics
    if (kRowsFirst<IO> ? !keys() || !queries() : !queries() || !keys())
        return GRKAN_ERR_LAUNCH;
    return hipGetLastError() == hipSuccess ? GRKAN_OK : GRKAN_ERR_LAUNCH;
}

} // namespace attention
} // namespace grkan

using namespace grkan;

extern "C" grkan_status_t grkan_attention_bwd(const grkan_attention_t *at, const void *out, const float *lse, const void *dout,
                                              int64_t dout_batch_stride, int64_t dout_token_stride, int64_t dout_head_stride, void *dq,
                                              void *dk, void *dv, void *workspace, size_t workspace_bytes, grkan_dtype_t io,
                                              void *hip_stream)
{
    attention::Args a;
    const grkan_status_t bad = attention::fill(at, io, &a);
    if (bad != GRKAN_OK)
        return bad;
    const bool rows = (int64_t)a.batch * a.rows > 0, keys = (int64_t)a.batch * a.keys > 0;
    if (!rows && !keys)
        return GRKAN_OK;
    if ((rows && (!out || !lse || !dout || !dq)) || (keys && (!dk || !dv)))
        return GRKAN_ERR_NULL;
    auto address = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if ((address(out) | address(dout) | address(dq) | address(dk) | address(dv)) % 16 != 0 || address(lse) % 4 != 0 ||
        (dout_batch_stride | dout_token_stride | dout_head_stride) % 8 != 0)
        return GRKAN_ERR_ALIGN;
    attention::BackPlan p = attention::back_plan(a, io);
    const size_t need = (p.stats + p.partial) * sizeof(float);
    if (need && (!workspace || workspace_bytes < need || address(workspace) % 16 != 0))
        return GRKAN_ERR_WORKSPACE;
    const size_t padded = (size_t)a.batch * (size_t)a.kv_heads * (size_t)p.keys.padded;
    for (attention::Args *to : {&p.keys, &p.queries}) {
        to->dout = attention::Operand{address(dout), dout_batch_stride * 2, dout_token_stride * 2, dout_head_stride * 2};
        to->even_q = attention::in_offsets(at->q_token_stride, at->q_head_stride, a.group);
        to->even_dout = attention::in_offsets(dout_token_stride, dout_head_stride, a.group);
        to->lse = const_cast<float *>(lse);
        to->row_lse = static_cast<float *>(workspace);
        to->row_delta = to->row_lse + padded;
        to->row_most = to->row_delta + padded;
        to->value_most = to->row_lse + p.value_most;
        to->partial = to->row_lse + p.stats;
        to->dk = static_cast<char *>(dk);
        to->dv = static_cast<char *>(dv);
    }
    p.keys.forward_out = p.queries.forward_out = address(out);
    p.queries.out = static_cast<char *>(dq);
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    return io == GRKAN_BF16 ? attention::backward<__bf16>(p, stream) : attention::backward<_Float16>(p, stream);
}
