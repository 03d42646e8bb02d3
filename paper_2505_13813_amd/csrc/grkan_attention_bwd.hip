// Cross attention on gfx950 (MI355X), backward.  With P recomputed from the rows' lse and D = dO V^T:
//
//     dV = P^T dO        S' = P (D - delta), delta = the row's sum of dO O        dQ = scale S' K        dK = scale S'^T Q
//
// Seven products as they stand (the scores and D twice), in two kernels, so that every gradient is summed by whoever owns it: no
// atomics, the same bits each time.  One has keys, walks the rows and keeps dK and dV; the other has rows, walks the keys and
// keeps dQ.  In both, as in the forward pass, the product that is contracted next is left in the registers as the operand of the next.
// A third, small one makes delta in front of them.
//
// float16: S' of a small upstream gradient would be below its range.  The products take 2^e S', with e such that the largest |dO| of
// the key head becomes 1/4 to 1/2 (2^e S' then stays below 65,504 for values of up to 1,000), and the sums are scaled back in float32.
#include <hip/hip_runtime.h>

#include "grkan_attention.h"

namespace grkan {
namespace attention {

constexpr int kRowTile = 64;

// Tiles of ROWS rows of the list: as TileLoads, but a row's place is its query's and its head's.
template <int DP, int ROWS, int WAVES> struct RowLoads {
    static constexpr int kChunks = DP / 8, kLoads = ROWS * kChunks / 64, kMine = (kLoads + WAVES - 1) / WAVES;
    static constexpr uint32_t kBytes = ROWS * DP * 2u;
    static_assert(kLoads % WAVES == 0, "");
    uint32_t row[kMine], chunk[kMine]; // chunk: its bytes, or ~0: no such channels
    int first;

    __device__ __forceinline__ RowLoads(int wave, int lane, int32_t dim) : first(wave)
    {
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t e = (uint32_t)(first + q * WAVES) * 64u + (uint32_t)lane;
            row[q] = e / kChunks;
            const uint32_t c = (e % kChunks) ^ swizzle<DP>(row[q]);
            chunk[q] = c * 8u < (uint32_t)dim ? c * 16u : ~0u;
        }
    }
    __device__ __forceinline__ void issue(const Operand &o, uint64_t base, uint32_t row0, const Args &a, uint32_t lds_at) const
    {
        const bool whole = a.group == 1 && a.dim == DP && (int64_t)row0 + ROWS <= a.rows;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const uint32_t to = lds_at + (uint32_t)(first + q * WAVES) * 1024u;
            if (whole) {
                load_to_lds(uniform_u64(base + (uint64_t)row0 * (uint64_t)o.token), row[q] * (uint32_t)o.token + chunk[q], to);
            } else {
                const bool there = (int64_t)row0 + row[q] < a.rows && chunk[q] != ~0u;
                const uint64_t at = base + (uint64_t)row_offset(row0 + row[q], (uint32_t)a.group, o.token, o.head) + chunk[q];
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

// delta, and copies of lse, of 64 rows for each workgroup: sixteen lanes a row, eight channels each.
template <typename IO> __global__ __launch_bounds__(256) void rows_kernel(const Args a)
{
    using MM = Matrix<IO>;
    __shared__ uint32_t most[4];
    const int32_t tiles = a.padded / kRowTile;
    const int32_t bh = (int32_t)blockIdx.x / tiles, tile = (int32_t)blockIdx.x - bh * tiles;
    const int32_t b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    const uint32_t lane16 = threadIdx.x & 15u;
    const int64_t heads_dim = (int64_t)a.kv_heads * a.group * a.dim;
    const uint64_t out = reinterpret_cast<uint64_t>(a.out) + 2u * (uint64_t)((int64_t)b * (a.rows / a.group) * heads_dim + (int64_t)kvh * a.group * a.dim);
    const uint64_t dout = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head);
    float largest = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t row = (uint32_t)tile * kRowTile + 16u * k + (threadIdx.x >> 4);
        const bool there = (int64_t)row < a.rows;
        float sum = 0.0f;
        if (there && 8u * lane16 < (uint32_t)a.dim) {
            const u32x4 o = gload16(out + 2u * (uint64_t)row_offset(row, (uint32_t)a.group, heads_dim, a.dim) + 16u * lane16, 0);
            const u32x4 d = gload16(dout + (uint64_t)row_offset(row, (uint32_t)a.group, a.dout.token, a.dout.head) + 16u * lane16, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = MM::first(d[j]), y = MM::second(d[j]);
                sum += x * MM::first(o[j]) + y * MM::second(o[j]);
                largest = fmaxf(largest, fmaxf(fabsf(x), fabsf(y)));
            }
        }
#pragma unroll
        for (int s = 8; s > 0; s /= 2)
            sum += __shfl_xor(sum, s);
        if (lane16 == 0) {
            const int64_t at = (int64_t)bh * a.padded + row;
            a.row_lse[at] = there ? a.lse[(int64_t)bh * a.rows + row] : __builtin_inff();
            a.row_delta[at] = sum;
        }
    }
    uint32_t bits = __builtin_bit_cast(uint32_t, largest);
#pragma unroll
    for (int s = 32; s > 0; s /= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)bits, s);
        bits = o > bits ? o : bits;
    }
    if ((threadIdx.x & 63) == 0)
        most[threadIdx.x >> 6] = bits;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w)
            bits = most[w] > bits ? most[w] : bits;
        a.row_most[(int64_t)bh * tiles + tile] = __builtin_bit_cast(float, bits);
    }
}

// 2^e for a key head (1 for bfloat16, and where dO is zero or not finite)
template <typename IO> __device__ __forceinline__ float gradient_scale(const Args &a, int32_t bh)
{
    if constexpr (sizeof(IO) == 2 && __is_same(IO, __bf16)) {
        return 1.0f;
    } else {
        const int32_t tiles = a.padded / kRowTile;
        uint32_t bits = 0;
        for (int32_t i = (int32_t)threadIdx.x & 63; i < tiles; i += 64) {
            const uint32_t o = __builtin_bit_cast(uint32_t, a.row_most[(int64_t)bh * tiles + i]);
            bits = o > bits ? o : bits;
        }
#pragma unroll
        for (int s = 32; s > 0; s /= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)bits, s);
            bits = o > bits ? o : bits;
        }
        // (dO is float16: its exponent is -24 .. 15)
        const int e = (int)(bits >> 23) - 127 + 2;
        return bits == 0 || e > 17 ? 1.0f : __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    }
}

template <typename IO_, int DP_, int B_, int WAVES_PER_SIMD_> struct BackShape {
    typedef IO_ IO;
    static constexpr int DP = DP_, B = B_, PER = WAVES_PER_SIMD_, kWaves = 4;
    static constexpr int kOwn = 32 * B * kWaves; // keys or rows of a workgroup
    static constexpr uint32_t kTile = kRowTile * DP * 2u;
    // key kernel: Q, dO, lse, delta of 64 rows; row kernel: K, V of 64 keys
    static constexpr uint32_t kKeyStage = 2 * kTile + 2 * kRowTile * 4u, kRowStage = 2 * kTile;
};

// dK and dV of 32 B keys a wavefront.
template <class SH> __global__ __launch_bounds__(256, SH::PER) void keys_kernel(const Args a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, B = SH::B, ND = DP / 32, NS = DP / 16;
    extern __shared__ __align__(256) char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = (uint32_t)lane & 31u, h = (uint32_t)lane >> 5;
    const int32_t item = work_item(a);
    if (item >= a.work)
        return;
    const int32_t per_head = a.key_tiles * a.splits;
    const int32_t bh = item / per_head, rest = item - bh * per_head;
    const int32_t key_tile = rest / a.splits, split = rest - key_tile * a.splits;
    const int32_t b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
    const int64_t count = keys_of(a, b);
    const int64_t key0 = (int64_t)key_tile * SH::kOwn + wave * 32 * B; // this wavefront's

    // ---- keys and values as second operands: lane l has key l mod 32, channels 16 s + 8 (l / 32) ..
    u32x4 k[B][NS], v[B][NS];
    bool valid[B];
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
#pragma unroll
    for (int kb = 0; kb < B; ++kb) {
        const int64_t key = key0 + 32 * kb + col;
        valid[kb] = key < count && (!a.mask || a.mask[(int64_t)b * a.mask_batch + key * a.mask_key] != 0);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool there = valid[kb] && channel < (uint32_t)a.dim;
            k[kb][s] = gload16(there ? k_base + (uint64_t)key * (uint64_t)a.k.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            v[kb][s] = gload16(there ? v_base + (uint64_t)key * (uint64_t)a.v.token + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
    }

    f32x16 dk[B][ND], dv[B][ND];
#pragma unroll
    for (int kb = 0; kb < B; ++kb)
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            dk[kb][d] = f32x16{};
            dv[kb][d] = f32x16{};
        }

    const RowLoads<DP, kRowTile, SH::kWaves> loads(wave, lane, a.dim);
    const RowOperand<DP> row_operand(lane);
    const ColumnOperand<DP> column_operand(lane);
    const uint64_t q_base = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head);
    const uint64_t d_base = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head);
    const int32_t tiles = a.padded / kRowTile;
    int32_t t0 = split * a.tiles_per_split, t1 = t0 + a.tiles_per_split;
    t1 = t1 < tiles ? t1 : tiles;
    // (no key of this workgroup is valid by its length: nothing to add)
    if ((int64_t)key_tile * SH::kOwn >= count)
        t1 = t0;
    const float up = gradient_scale<IO>(a, bh), c = a.c;

    auto issue = [&](int32_t t, uint32_t stage) {
        const uint32_t row0 = (uint32_t)t * kRowTile;
        loads.issue(a.q, q_base, row0, a, stage);
        loads.issue(a.dout, d_base, row0, a, stage + SH::kTile);
        if (wave < 2) {
            const float *const from = (wave ? a.row_delta : a.row_lse) + (int64_t)bh * a.padded + row0;
            load_words_to_lds(uniform_u64(reinterpret_cast<uint64_t>(from)), (uint32_t)lane * 4u, stage + 2 * SH::kTile + (uint32_t)wave * kRowTile * 4u);
        }
    };

    uint32_t at = 0;
    if (t0 < t1)
        issue(t0, lds0);
    for (int32_t t = t0; t < t1; ++t) {
        wait_loads<0>();
        barrier();
        if (t + 1 < t1)
            issue(t + 1, lds0 + (at ^ SH::kKeyStage));
        const uint32_t stage = lds0 + at, stats = stage + 2 * SH::kTile;
#pragma unroll
        for (int rb = 0; rb < kRowTile / 32; ++rb) {
            f32x16 s[B], d[B];
#pragma unroll
            for (int kb = 0; kb < B; ++kb) {
                s[kb] = f32x16{};
                d[kb] = f32x16{};
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const u32x4 q = row_operand.read(stage, rb, st);
#pragma unroll
                for (int kb = 0; kb < B; ++kb)
                    s[kb] = MM::multiply(q, k[kb][st], s[kb]);
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const u32x4 o = row_operand.read(stage + SH::kTile, rb, st);
#pragma unroll
                for (int kb = 0; kb < B; ++kb)
                    d[kb] = MM::multiply(o, v[kb][st], d[kb]);
            }
            uint32_t p[B][8], g[B][8];
#pragma unroll
            for (int quad = 0; quad < 4; ++quad) {
                const uint32_t place = stats + (32u * rb + 8u * quad + 4u * h) * 4u;
                const f32x4 lse = __builtin_bit_cast(f32x4, lds_read16(place)), delta = __builtin_bit_cast(f32x4, lds_read16(place + kRowTile * 4u));
#pragma unroll
                for (int kb = 0; kb < B; ++kb) {
                    float x[4], y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = __builtin_amdgcn_exp2f(fmaf(s[kb][4 * quad + j], c, -lse[j]));
                        y[j] = x[j] * fmaf(d[kb][4 * quad + j], up, -delta[j] * up);
                    }
                    p[kb][2 * quad] = MM::two(x[0], x[1]);
                    p[kb][2 * quad + 1] = MM::two(x[2], x[3]);
                    g[kb][2 * quad] = MM::two(y[0], y[1]);
                    g[kb][2 * quad + 1] = MM::two(y[2], y[3]);
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int part = 0; part < ND; ++part) {
                    const u32x4 o = column_operand.read(stage + SH::kTile, rb, half, part), q = column_operand.read(stage, rb, half, part);
#pragma unroll
                    for (int kb = 0; kb < B; ++kb) {
                        u32x4 w, z;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            w[j] = p[kb][4 * half + j];
                            z[j] = g[kb][4 * half + j];
                        }
                        dv[kb][part] = MM::multiply(o, w, dv[kb][part]);
                        dk[kb][part] = MM::multiply(q, z, dk[kb][part]);
                    }
                }
        }
        at ^= SH::kKeyStage;
    }

    const float by = a.scale / up;
#pragma unroll
    for (int kb = 0; kb < B; ++kb) {
        const int64_t key = key0 + 32 * kb + col;
        if (key >= a.keys)
            continue;
        const int64_t line = ((int64_t)b * a.keys + key) * a.kv_heads + kvh;
        const int64_t all = (int64_t)a.batch * a.keys * a.kv_heads;
#pragma unroll
        for (int part = 0; part < ND; ++part)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int channel = 32 * part + 8 * g + 4 * (int)h;
                if (channel < a.dim) {
                    f32x4 x, y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = valid[kb] ? dk[kb][part][4 * g + j] * by : 0.0f;
                        y[j] = valid[kb] ? dv[kb][part][4 * g + j] : 0.0f;
                    }
                    if (a.splits == 1) {
                        u32x2 w, z;
                        w[0] = MM::two(x[0], x[1]);
                        w[1] = MM::two(x[2], x[3]);
                        z[0] = MM::two(y[0], y[1]);
                        z[1] = MM::two(y[2], y[3]);
                        *reinterpret_cast<u32x2 *>(a.dk + (line * a.dim + channel) * 2) = w;
                        *reinterpret_cast<u32x2 *>(a.dv + (line * a.dim + channel) * 2) = z;
                    } else {
                        float *const to = a.partial + ((int64_t)split * all + line) * a.dim + channel;
                        *reinterpret_cast<f32x4 *>(to) = x;
                        *reinterpret_cast<f32x4 *>(to + (int64_t)a.splits * all * a.dim) = y;
                    }
                }
            }
    }
}

// dQ of 32 B rows a wavefront.
template <class SH> __global__ __launch_bounds__(256, SH::PER) void queries_kernel(const Args a)
{
    using IO = typename SH::IO;
    using MM = Matrix<IO>;
    constexpr int DP = SH::DP, B = SH::B, ND = DP / 32, NS = DP / 16, KT = kRowTile;
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
    const int64_t count = keys_of(a, b);
    const int32_t tiles = (int32_t)((count + KT - 1) / KT);
    int32_t t0 = split * a.tiles_per_split, t1 = t0 + a.tiles_per_split;
    t1 = t1 < tiles ? t1 : tiles;

    const uint32_t row0 = (uint32_t)row_tile * SH::kOwn + (uint32_t)wave * 32u * B;
    const uint64_t q_base = a.q.at + (uint64_t)(b * a.q.batch + (int64_t)kvh * a.group * a.q.head);
    const uint64_t d_base = a.dout.at + (uint64_t)(b * a.dout.batch + (int64_t)kvh * a.group * a.dout.head);
    const float up = gradient_scale<IO>(a, bh), c = a.c;
    u32x4 q[B][NS], o[B][NS];
    float lse[B], delta[B];
    f32x16 dq[B][ND];
#pragma unroll
    for (int rb = 0; rb < B; ++rb) {
        const uint32_t row = row0 + 32u * rb + col;
        const bool row_there = (int64_t)row < a.rows;
        const int64_t qo = row_offset(row, (uint32_t)a.group, a.q.token, a.q.head), oo = row_offset(row, (uint32_t)a.group, a.dout.token, a.dout.head);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t channel = 16u * s + 8u * h;
            const bool there = row_there && channel < (uint32_t)a.dim;
            q[rb][s] = gload16(there ? q_base + (uint64_t)qo + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
            o[rb][s] = gload16(there ? d_base + (uint64_t)oo + channel * 2u : reinterpret_cast<uint64_t>(kZeros), 0);
        }
        lse[rb] = row_there ? a.row_lse[(int64_t)bh * a.padded + row] : __builtin_inff();
        delta[rb] = row_there ? a.row_delta[(int64_t)bh * a.padded + row] * up : 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
            dq[rb][d] = f32x16{};
    }

    const TileLoads<DP, KT, SH::kWaves> k_loads(wave, lane, a.k.token, a.dim), v_loads(wave, lane, a.v.token, a.dim);
    const RowOperand<DP> row_operand(lane);
    const ColumnOperand<DP> column_operand(lane);
    const uint64_t k_base = a.k.at + (uint64_t)(b * a.k.batch + kvh * a.k.head), v_base = a.v.at + (uint64_t)(b * a.v.batch + kvh * a.v.head);
    ValidKeys valid(a, b, count);
    auto issue = [&](int32_t t, uint64_t word, uint32_t stage) {
        const bool whole = word == ~(uint64_t)0 && a.dim == DP;
        k_loads.issue(k_base + (uint64_t)t * KT * (uint64_t)a.k.token, word, whole, stage);
        v_loads.issue(v_base + (uint64_t)t * KT * (uint64_t)a.v.token, word, whole, stage + SH::kTile);
    };

    uint32_t at = 0;
    uint64_t word = 0;
    if (t0 < t1) {
        word = valid.word(t0);
        issue(t0, word, lds0);
    }
    for (int32_t t = t0; t < t1; ++t) {
        const uint64_t next = t + 1 < t1 ? valid.word(t + 1) : 0;
        wait_loads<0>();
        barrier();
        if (t + 1 < t1)
            issue(t + 1, next, lds0 + (at ^ SH::kRowStage));
        const uint32_t stage = lds0 + at;
#pragma unroll
        for (int kb = 0; kb < KT / 32; ++kb) {
            f32x16 s[B], d[B];
#pragma unroll
            for (int rb = 0; rb < B; ++rb) {
                s[rb] = f32x16{};
                d[rb] = f32x16{};
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const u32x4 k = row_operand.read(stage, kb, st);
#pragma unroll
                for (int rb = 0; rb < B; ++rb)
                    s[rb] = MM::multiply(k, q[rb][st], s[rb]);
            }
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const u32x4 v = row_operand.read(stage + SH::kTile, kb, st);
#pragma unroll
                for (int rb = 0; rb < B; ++rb)
                    d[rb] = MM::multiply(v, o[rb][st], d[rb]);
            }
            uint32_t g[B][8];
#pragma unroll
            for (int rb = 0; rb < B; ++rb) {
                float y[16];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    y[i] = __builtin_amdgcn_exp2f(fmaf(s[rb][i], c, -lse[rb])) * fmaf(d[rb][i], up, -delta[rb]);
                if (word != ~(uint64_t)0) {
                    const uint32_t bits = (uint32_t)((word >> (32 * kb)) >> (4u * h));
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        y[i] = (bits >> (8 * (i / 4) + i % 4)) & 1u ? y[i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 16; i += 2)
                    g[rb][i / 2] = MM::two(y[i], y[i + 1]);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int part = 0; part < ND; ++part) {
                    const u32x4 k = column_operand.read(stage, kb, half, part);
#pragma unroll
                    for (int rb = 0; rb < B; ++rb) {
                        u32x4 z;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            z[j] = g[rb][4 * half + j];
                        dq[rb][part] = MM::multiply(k, z, dq[rb][part]);
                    }
                }
        }
        at ^= SH::kRowStage;
        word = next;
    }

    const float by = a.scale / up;
    const int64_t heads = (int64_t)a.kv_heads * a.group, all = (int64_t)a.batch * a.kv_heads * a.rows;
#pragma unroll
    for (int rb = 0; rb < B; ++rb) {
        const uint32_t row = row0 + 32u * rb + col;
        if ((int64_t)row >= a.rows)
            continue;
        const int64_t line = (int64_t)b * (a.rows / a.group) * heads + (int64_t)kvh * a.group + row_offset(row, (uint32_t)a.group, heads, 1);
#pragma unroll
        for (int part = 0; part < ND; ++part)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int channel = 32 * part + 8 * g + 4 * (int)h;
                if (channel < a.dim) {
                    f32x4 x;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        x[j] = dq[rb][part][4 * g + j] * by;
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
    int own_keys, own_rows;
    size_t keys_lds, queries_lds;
};
template <class KS, class QS> static BackVariant back_variant()
{
    return BackVariant{keys_kernel<KS>, queries_kernel<QS>, KS::kOwn, QS::kOwn, 2 * (size_t)KS::kKeyStage, 2 * (size_t)QS::kRowStage};
}
template <typename IO> static BackVariant pick(int32_t dim)
{
    if (dim <= 32)
        return back_variant<BackShape<IO, 32, 1, 2>, BackShape<IO, 32, 1, 2>>();
    if (dim <= 64)
        return back_variant<BackShape<IO, 64, 1, 2>, BackShape<IO, 64, 1, 2>>();
    if (dim <= 96)
        return back_variant<BackShape<IO, 96, 1, 2>, BackShape<IO, 96, 1, 2>>();
    return back_variant<BackShape<IO, 128, 1, 1>, BackShape<IO, 128, 1, 2>>();
}

// How many workgroups share the walk of one: enough to give each compute unit two, four tiles each at least.
static void split(int64_t base, int64_t tiles, Args &a)
{
    int64_t splits = base > 0 && base < 384 ? 512 / base : 1;
    splits = splits < tiles / 4 ? splits : tiles / 4;
    splits = splits > 1 ? splits : 1;
    const int64_t per = (tiles + splits - 1) / splits;
    a.tiles_per_split = (int32_t)(per > 1 ? per : 1);
    a.splits = (int32_t)((tiles + a.tiles_per_split - 1) / a.tiles_per_split);
    if (a.splits < 1)
        a.splits = 1;
}

struct BackPlan {
    BackVariant v;
    Args keys, queries;
    size_t stats, partial; // elements of the workspace
};

static BackPlan back_plan(const Args &a, grkan_dtype_t io)
{
    BackPlan p;
    p.v = io == GRKAN_BF16 ? pick<__bf16>(a.dim) : pick<_Float16>(a.dim);
    p.keys = p.queries = a;
    const int64_t heads = (int64_t)a.batch * a.kv_heads;
    const int32_t padded = (int32_t)((a.rows + kRowTile - 1) / kRowTile) * kRowTile;
    p.keys.padded = p.queries.padded = padded;
    p.keys.key_tiles = (int32_t)((a.keys + p.v.own_keys - 1) / p.v.own_keys);
    p.queries.row_tiles = (int32_t)((a.rows + p.v.own_rows - 1) / p.v.own_rows);
    split(heads * p.keys.key_tiles, padded / kRowTile, p.keys);
    split(heads * p.queries.row_tiles, (a.keys + kRowTile - 1) / kRowTile, p.queries);
    p.stats = (size_t)heads * (size_t)padded * 2 + (((size_t)heads * (size_t)(padded / kRowTile) + 3) & ~(size_t)3);
    // (one after the other: they share the memory)
    const size_t of_keys = p.keys.splits > 1 ? 2 * (size_t)p.keys.splits * (size_t)heads * (size_t)a.keys * (size_t)a.dim : 0;
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
    const int64_t key_work = heads * k.key_tiles * k.splits, row_work = heads * q.row_tiles * q.splits;
    const int64_t key_elements = (int64_t)k.batch * k.keys * k.kv_heads * k.dim, row_elements = heads * k.rows * k.dim;
    const int64_t key_blocks = (key_elements / 8 + 255) / 256, row_blocks = (row_elements / 8 + 255) / 256;
    if (rows_grid > INT32_MAX || key_work > INT32_MAX - 8 || row_work > INT32_MAX - 8 || (k.splits > 1 && key_blocks > INT32_MAX) ||
        (q.splits > 1 && row_blocks > INT32_MAX))
        return GRKAN_ERR_UNSUPPORTED;
    if (!allow_lds(reinterpret_cast<const void *>(p.v.keys), p.v.keys_lds) || !allow_lds(reinterpret_cast<const void *>(p.v.queries), p.v.queries_lds))
        return GRKAN_ERR_LAUNCH;
    if (rows_grid > 0)
        rows_kernel<IO><<<dim3((unsigned)rows_grid), 256, 0, stream>>>(k);
    if (key_work > 0) {
        k.work = (int32_t)key_work;
        k.per_xcd = (int32_t)((key_work + 7) / 8);
        void *args[] = {&k};
        if (hipLaunchKernel(reinterpret_cast<const void *>(p.v.keys), dim3((unsigned)k.per_xcd * 8u), dim3(256), args, p.v.keys_lds, stream) != hipSuccess)
            return GRKAN_ERR_LAUNCH;
        if (k.splits > 1) {
            sum_kernel<IO><<<dim3((unsigned)key_blocks), 256, 0, stream>>>(k.partial, k.splits, key_elements, k.dk);
            sum_kernel<IO><<<dim3((unsigned)key_blocks), 256, 0, stream>>>(k.partial + (int64_t)k.splits * key_elements, k.splits, key_elements, k.dv);
        }
    }
    if (row_work > 0) {
        q.work = (int32_t)row_work;
        q.per_xcd = (int32_t)((row_work + 7) / 8);
        void *args[] = {&q};
        if (hipLaunchKernel(reinterpret_cast<const void *>(p.v.queries), dim3((unsigned)q.per_xcd * 8u), dim3(256), args, p.v.queries_lds, stream) != hipSuccess)
            return GRKAN_ERR_LAUNCH;
        if (q.splits > 1)
            sum_kernel<IO><<<dim3((unsigned)row_blocks), 256, 0, stream>>>(q.partial, q.splits, row_elements, q.out);
    }
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
    if (dout_token_stride < 0 || dout_token_stride > (((int64_t)1 << 31) - 512) / 128)
        return GRKAN_ERR_UNSUPPORTED;
    attention::BackPlan p = attention::back_plan(a, io);
    const size_t need = (p.stats + p.partial) * sizeof(float);
    if (need && (!workspace || workspace_bytes < need || address(workspace) % 16 != 0))
        return GRKAN_ERR_WORKSPACE;
    const size_t padded = (size_t)a.batch * (size_t)a.kv_heads * (size_t)p.keys.padded;
    for (attention::Args *to : {&p.keys, &p.queries}) {
        to->dout = attention::Operand{address(dout), dout_batch_stride * 2, dout_token_stride * 2, dout_head_stride * 2};
        to->lse = const_cast<float *>(lse);
        to->row_lse = static_cast<float *>(workspace);
        to->row_delta = to->row_lse + padded;
        to->row_most = to->row_delta + padded;
        to->partial = to->row_lse + p.stats;
        to->dk = static_cast<char *>(dk);
        to->dv = static_cast<char *>(dv);
    }
    p.keys.out = static_cast<char *>(const_cast<void *>(out)); // (read by the rows' kernel)
    p.queries.out = static_cast<char *>(dq);
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    return io == GRKAN_BF16 ? attention::backward<__bf16>(p, stream) : attention::backward<_Float16>(p, stream);
}
