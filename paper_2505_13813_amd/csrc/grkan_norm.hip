// Root-mean-square norm with the residual's addition on gfx950 (MI355X), forward, to 8 bits, and backward.
//
//     h = x + r,  s = (mean h^2 + eps)^(-1/2),  y = h s w
//     dx = s (g - n mean(g n)) + dh  with g = dy w, n = h s          dw = sum over rows of dy n
//
// Bound by memory: 16 operations an element against 8 bytes (forward, 16-bit types) or 8 more (backward).  So a row is read once and
// stays in registers from the sum of squares to the store: one wavefront has a row of up to 2,048 elements (1,024 in float32), four
// wavefronts one of up to 8,192 (4,096), sixteen a longer one.  A row whose length is no multiple of the vector ends in a vector that
// repeats elements of the one before: they are stored twice with the same value and counted once.  (25,216 x 768 in bfloat16 with a
// residual: forward 28.5 us = 5.4 TB/s, where a large copy reaches 5.5; 16,384 x 4096 to 8 bits 82 us = 5.7 TB/s.
// float32, 4,096 x 8192 with a residual, sixteen wavefronts: forward 94 us = 5.7 TB/s, backward, which spills two registers there, 112 = 4.8; 8,192 x 4096 with
// four, which does not spill, 88 and 115.)
//
// The weights' gradient is a sum over rows: a lane has the same columns in every row it visits and keeps their sums in registers; each
// workgroup leaves one row of sums in the workspace, and a second launch adds those in a fixed order.  (25,216 x 768: 28 to 32 us for
// 155 MB, a part of them in the last-level cache, and 4 for the second launch; atomics would change the sums' order.)
#include <hip/hip_runtime.h>

#include "../../include/grkan_transformer.h"
#include "grkan_vector.h"

namespace grkan {
namespace norm {

using namespace vec;

constexpr int kMaxWidth = 16384;
constexpr float kMost8 = 448.0f;

struct Args {
    const void *x, *residual, *weight; // backward: x is h, residual dh
    const void *dy;
    void *h, *y;                       // backward: y is dx
    float *scale;
    float *partial;
    int64_t rows, x_stride, residual_stride, dy_stride;
    int32_t D;
    float eps;
};

// WAVES wavefronts have a row, NV vectors of it a lane; workgroups of 256 lanes or, with more than four wavefronts to a row, one row.
template <typename IO_, int VEC_, int WAVES_, int NV_> struct Shape {
    typedef IO_ IO;
    static constexpr int VEC = VEC_, WAVES = WAVES_, NV = NV_;
    static constexpr int kThreads = WAVES > 4 ? 64 * WAVES : 256, kRows = kThreads / (64 * WAVES);
    static constexpr int kWidth = 64 * WAVES * VEC * NV;
};

// sums (and, in integers, maxima) over the WAVES wavefronts of a row; `slot` alternates so that one barrier is enough
template <class SH> __device__ __forceinline__ float row_sum(float v, float *shared, int &slot)
{
    v = wave_sum(v);
    if constexpr (SH::WAVES > 1) {
        float *const at = shared + slot * SH::WAVES;
        slot ^= 1;
        if ((threadIdx.x & 63) == 0)
            at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < SH::WAVES; ++w)
            v += at[w];
    }
    return v;
}
template <class SH> __device__ __forceinline__ uint32_t row_max(uint32_t v, float *shared, int &slot)
{
    v = wave_max(v);
    if constexpr (SH::WAVES > 1) {
        uint32_t *const at = reinterpret_cast<uint32_t *>(shared) + slot * SH::WAVES;
        slot ^= 1;
        if ((threadIdx.x & 63) == 0)
            at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < SH::WAVES; ++w)
            v = at[w] > v ? at[w] : v;
    }
    return v;
}

// Where a lane's vector i of a row starts, and how many of its first elements belong to the vector before; the vector is not
// there at all if own == VEC.
template <class SH> struct Columns {
    int32_t at[SH::NV], own[SH::NV];
    __device__ __forceinline__ explicit Columns(int32_t D)
    {
        const int32_t lane = (int32_t)threadIdx.x % (64 * SH::WAVES);
#pragma unroll
        for (int i = 0; i < SH::NV; ++i) {
            const int32_t c = (i * 64 * SH::WAVES + lane) * SH::VEC, last = D - SH::VEC;
            at[i] = c < last ? c : last;
            own[i] = c >= D ? SH::VEC : c - at[i];
        }
    }
};

template <class SH, typename W> __device__ __forceinline__ void load_weights(const void *weight, const Columns<SH> &cols, float (&w)[SH::NV][SH::VEC])
{
#pragma unroll
    for (int i = 0; i < SH::NV; ++i)
        widen<W, SH::VEC>(load<W, SH::VEC>(static_cast<const W *>(weight) + cols.at[i]), w[i]);
}

template <class SH, typename W, bool RESIDUAL, bool EIGHT> __global__ __launch_bounds__(SH::kThreads) void forward_kernel(const Args a)
{
    using IO = typename SH::IO;
    constexpr int VEC = SH::VEC, NV = SH::NV;
    typedef typename Raw<IO, VEC>::type raw_t;
    __shared__ float shared[2 * SH::WAVES];
    int slot = 0;
    const Columns<SH> cols(a.D);
    float w[NV][VEC];
    load_weights<SH, W>(a.weight, cols, w);
    const int sub = SH::kRows > 1 ? (int)threadIdx.x >> 6 : 0;
    for (int64_t row = (int64_t)blockIdx.x * SH::kRows + sub; row < a.rows; row += (int64_t)gridDim.x * SH::kRows) {
        const IO *const x = static_cast<const IO *>(a.x) + row * a.x_stride;
        const IO *const r = RESIDUAL ? static_cast<const IO *>(a.residual) + row * a.residual_stride : nullptr;
        raw_t xs[NV], rs[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                xs[i] = load<IO, VEC>(x + cols.at[i]);
                if (RESIDUAL)
                    rs[i] = load<IO, VEC>(r + cols.at[i]);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                float f[VEC];
                widen<IO, VEC>(xs[i], f);
                if (RESIDUAL) {
                    float g[VEC];
                    widen<IO, VEC>(rs[i], g);
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        f[e] += g[e];
                    xs[i] = narrow<IO, VEC>(f);
                    widen<IO, VEC>(xs[i], f);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    sum += e >= cols.own[i] ? f[e] * f[e] : 0.0f;
            }
        }
        sum = row_sum<SH>(sum, shared, slot);
        const float s = rsqrtf(sum / (float)a.D + a.eps);
        // To 8 bits: y / scale = 448 h w / max |h w| does not depend on s, and of 16-bit numbers the product h w is exact; the factor's
        // remainder is kept too, so that nothing but the last step rounds.  (h in units of s rounded to a power of 2, so that its products
        // stay in range.)
        float unit = 1.0f, factor = 0.0f, remainder = 0.0f;
        if constexpr (EIGHT) {
            // (s is infinite for a row of zeros, where eps is 0)
            unit = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, fminf(s, 0x1p126f)) & 0x7f800000u);
            // magnitudes as whole numbers: a NaN is the largest
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (cols.own[i] < VEC) {
                    float f[VEC];
                    widen<IO, VEC>(xs[i], f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const uint32_t b = __builtin_bit_cast(uint32_t, f[e] * unit * w[i][e]) & 0x7fffffffu;
                        most = b > most ? b : most;
                    }
                }
            }
            const float largest = __builtin_bit_cast(float, row_max<SH>(most, shared, slot));
            const float amax = largest == 0.0f && s == __builtin_inff() ? 0.0f : largest * (s / unit);
            const float scale = amax < __builtin_inff() ? amax / kMost8 : __builtin_nanf("");
            if (scale != scale) {
                factor = scale;
            } else if (largest > 0.0f) {
                if (largest < 0x1p-80f) // (448 / largest would overflow for the smallest)
                    unit *= 0x1p100f;
                const float m = largest < 0x1p-80f ? largest * 0x1p100f : largest;
                factor = kMost8 / m;
                remainder = fmaf(-factor, m, kMost8) / m;
            }
            if (threadIdx.x % (64 * SH::WAVES) == 0)
                a.scale[row] = scale;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                const int64_t at = row * a.D + cols.at[i];
                if (RESIDUAL)
                    store<IO, VEC>(static_cast<IO *>(a.h) + at, xs[i]);
                float f[VEC];
                widen<IO, VEC>(xs[i], f);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    f[e] = EIGHT ? f[e] * unit * w[i][e] : f[e] * s * w[i][e];
                if constexpr (EIGHT) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        f[e] = fmaf(f[e], factor, f[e] * remainder);
                    typedef uint8_t bytes_t __attribute__((ext_vector_type(VEC), aligned(1)));
                    uint8_t b[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        const uint32_t two = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[e], e + 1 < VEC ? f[e + 1] : 0.0f, 0, false);
                        b[e] = (uint8_t)two;
                        if (e + 1 < VEC)
                            b[e + 1] = (uint8_t)(two >> 8);
                    }
                    uint8_t *const p = static_cast<uint8_t *>(a.y) + at;
                    if constexpr (VEC == 1) {
                        *p = b[0];
                    } else {
                        bytes_t v;
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            v[e] = b[e];
                        *reinterpret_cast<bytes_t *>(p) = v;
                    }
                } else {
                    store<IO, VEC>(static_cast<IO *>(a.y) + at, narrow<IO, VEC>(f));
                }
            }
        }
    }
}

template <class SH, typename W, bool RESIDUAL> __global__ __launch_bounds__(SH::kThreads) void backward_kernel(const Args a)
{
    using IO = typename SH::IO;
    constexpr int VEC = SH::VEC, NV = SH::NV;
    typedef typename Raw<IO, VEC>::type raw_t;
    __shared__ float shared[4 * SH::WAVES];
    __shared__ float joined[SH::kRows > 1 ? SH::kWidth : 1];
    int slot = 0;
    const Columns<SH> cols(a.D);
    float w[NV][VEC], dw[NV][VEC];
    load_weights<SH, W>(a.weight, cols, w);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            dw[i][e] = 0.0f;
    const int sub = SH::kRows > 1 ? (int)threadIdx.x >> 6 : 0;
    for (int64_t row = (int64_t)blockIdx.x * SH::kRows + sub; row < a.rows; row += (int64_t)gridDim.x * SH::kRows) {
        const IO *const h = static_cast<const IO *>(a.x) + row * a.x_stride;
        const IO *const dy = static_cast<const IO *>(a.dy) + row * a.dy_stride;
        const IO *const dh = RESIDUAL ? static_cast<const IO *>(a.residual) + row * a.residual_stride : nullptr;
        raw_t hs[NV], ds[NV], rs[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                hs[i] = load<IO, VEC>(h + cols.at[i]);
                ds[i] = load<IO, VEC>(dy + cols.at[i]);
                if (RESIDUAL)
                    rs[i] = load<IO, VEC>(dh + cols.at[i]);
            }
        }
        float squares = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                float f[VEC], g[VEC];
                widen<IO, VEC>(hs[i], f);
                widen<IO, VEC>(ds[i], g);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    squares += e >= cols.own[i] ? f[e] * f[e] : 0.0f;
                    along += e >= cols.own[i] ? g[e] * w[i][e] * f[e] : 0.0f;
                }
            }
        }
        squares = wave_sum(squares);
        along = wave_sum(along);
        if constexpr (SH::WAVES > 1) {
            float *const at = shared + slot * 2 * SH::WAVES;
            slot ^= 1;
            if ((threadIdx.x & 63) == 0) {
                at[threadIdx.x >> 6] = squares;
                at[SH::WAVES + (threadIdx.x >> 6)] = along;
            }
            __syncthreads();
            squares = along = 0.0f;
#pragma unroll
            for (int v = 0; v < SH::WAVES; ++v) {
                squares += at[v];
                along += at[SH::WAVES + v];
            }
        }
        const float s = rsqrtf(squares / (float)a.D + a.eps);
        const float c = along * s * s / (float)a.D; // of h: s n mean(g n) = h s c
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (cols.own[i] < VEC) {
                float f[VEC], g[VEC], d[VEC];
                widen<IO, VEC>(hs[i], f);
                widen<IO, VEC>(ds[i], g);
                if (RESIDUAL)
                    widen<IO, VEC>(rs[i], d);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    dw[i][e] += e >= cols.own[i] ? g[e] * (f[e] * s) : 0.0f;
                    const float dx = s * (g[e] * w[i][e] - f[e] * c);
                    f[e] = RESIDUAL ? d[e] + dx : dx;
                }
                store<IO, VEC>(static_cast<IO *>(a.y) + row * a.D + cols.at[i], narrow<IO, VEC>(f));
            }
        }
    }
    // one row of sums for each workgroup: with a row to each wavefront, wavefront by wavefront
    float *const out = a.partial + (int64_t)blockIdx.x * a.D;
    if constexpr (SH::kRows > 1) {
        for (int turn = 0; turn < SH::kRows; ++turn) {
            if (sub == turn) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if (e >= cols.own[i]) {
                            float *const p = joined + cols.at[i] + e;
                            *p = turn ? *p + dw[i][e] : dw[i][e];
                        }
                    }
            }
            __syncthreads();
        }
        for (int32_t c = (int32_t)threadIdx.x; c < a.D; c += SH::kThreads)
            out[c] = joined[c];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e >= cols.own[i])
                    out[cols.at[i] + e] = dw[i][e];
    }
}

// dw[c] = the sum of column c of the workspace's rows: sixteen columns to a workgroup, whose 64 slices of rows are added in order
template <typename W> __global__ __launch_bounds__(1024) void columns_kernel(const float *partial, int32_t count, int32_t D, W *dw)
{
    __shared__ float part[64][17];
    const int32_t lane = (int32_t)threadIdx.x & 15, slice = (int32_t)threadIdx.x >> 4;
    const int32_t c = (int32_t)blockIdx.x * 16 + lane;
    float v = 0.0f;
    if (c < D) {
#pragma unroll 16
        for (int32_t r = slice; r < count; r += 64)
            v += partial[(int64_t)r * D + c];
    }
    part[slice][lane] = v;
    __syncthreads();
    if (slice == 0 && c < D) {
        v = 0.0f;
        for (int i = 0; i < 64; ++i)
            v += part[i][lane];
        dw[c] = (W)v;
    }
}

typedef void (*Kernel)(Args);
struct Variant {
    Kernel kernel;
    int threads, rows; // of a workgroup
};

// which: 0 forward, 1 to 8 bits, 2 backward
template <class SH, typename W> static Variant pick(int which, bool residual)
{
    Kernel k;
    if (which == 0)
        k = residual ? forward_kernel<SH, W, true, false> : forward_kernel<SH, W, false, false>;
    else if (which == 1)
        k = residual ? forward_kernel<SH, W, true, true> : forward_kernel<SH, W, false, true>;
    else
        k = residual ? backward_kernel<SH, W, true> : backward_kernel<SH, W, false>;
    return Variant{k, SH::kThreads, SH::kRows};
}

// The fewest wavefronts that hold a row in registers.
template <typename IO, typename W> static Variant choose(int32_t D, int which, bool residual)
{
    constexpr int V = 16 / sizeof(IO); // 16-byte vectors
    if (D < V)
        return pick<Shape<IO, 1, 1, 1>, W>(which, residual);
    if (D <= 64 * V)
        return pick<Shape<IO, V, 1, 1>, W>(which, residual);
    if (D <= 128 * V)
        return pick<Shape<IO, V, 1, 2>, W>(which, residual);
    if (D <= 256 * V)
        return pick<Shape<IO, V, 1, 4>, W>(which, residual);
    if (D <= 512 * V)
        return pick<Shape<IO, V, 4, 2>, W>(which, residual);
    if (D <= 1024 * V)
        return pick<Shape<IO, V, 4, 4>, W>(which, residual);
    return pick<Shape<IO, V, 16, 16 / V>, W>(which, residual);
}

static Variant choose(int32_t D, grkan_dtype_t io, grkan_dtype_t wt, int which, bool residual)
{
    if (io == GRKAN_F32)
        return choose<float, float>(D, which, residual);
    if (io == GRKAN_BF16)
        return wt == GRKAN_F32 ? choose<__bf16, float>(D, which, residual) : choose<__bf16, __bf16>(D, which, residual);
    return wt == GRKAN_F32 ? choose<_Float16, float>(D, which, residual) : choose<_Float16, _Float16>(D, which, residual);
}

// Workgroups.  Forward: nearly one for each row or four (of a row below a KB two or more, which the start of a workgroup is worth); us with
// 2,048 / 16,384 of them: 25,216 x 768 in bfloat16 with a residual 32.7 / 28.0, 16,384 x 4096 103 / 87, 40,000 x 768 in float32 88 / 82;
// 60,000 x 192 20.6 / 24.6.  Backward: each keeps its columns' sums for all the rows it visits, and writes them; 512 / 1,024 / 1,536 of them:
// 25,216 x 768 34 / 27 / 34, 16,384 x 4096 116 / 87 / 104, 8,192 x 8192 115 / 124 / 134.
static int64_t grid_of(const Variant &v, int64_t rows, int32_t D, grkan_dtype_t io, bool backward)
{
    const int64_t bytes = (int64_t)D * (io == GRKAN_F32 ? 4 : 2);
    const int64_t most = backward ? (v.threads > 256 ? 256 : bytes > 8192 ? 512 : 1024) : bytes < 1024 ? 2048 : 16384;
    const int64_t need = (rows + v.rows - 1) / v.rows;
    return need < most ? need : most;
}

static grkan_status_t check(int64_t rows, int32_t D, grkan_dtype_t io, grkan_dtype_t wt)
{
    if (rows < 0 || D <= 0)
        return GRKAN_ERR_SHAPE;
    if (io != GRKAN_F32 && io != GRKAN_BF16 && io != GRKAN_F16)
        return GRKAN_ERR_DTYPE;
    if (wt != GRKAN_F32 && wt != io)
        return GRKAN_ERR_DTYPE;
    return D > kMaxWidth || rows > (int64_t)1 << 40 ? GRKAN_ERR_UNSUPPORTED : GRKAN_OK;
}

static bool misaligned(const void *p, grkan_dtype_t t) { return reinterpret_cast<uintptr_t>(p) % (t == GRKAN_F32 ? 4 : 2) != 0; }

} // namespace norm
} // namespace grkan

using namespace grkan;

extern "C" grkan_status_t grkan_rms_norm_fwd(const void *x, const void *residual, const void *weight, void *h, void *y, float *scale,
                                             int64_t rows, int32_t D, int64_t x_stride, int64_t residual_stride, float eps,
                                             grkan_dtype_t io, grkan_dtype_t weight_dtype, void *hip_stream)
{
    const grkan_status_t bad = norm::check(rows, D, io, weight_dtype);
    if (bad != GRKAN_OK)
        return bad;
    if (!weight || (rows > 0 && (!x || !y || (residual && !h))))
        return GRKAN_ERR_NULL;
    if (norm::misaligned(x, io) || norm::misaligned(residual, io) || norm::misaligned(h, io) || (!scale && norm::misaligned(y, io)) ||
        norm::misaligned(weight, weight_dtype) || norm::misaligned(scale, GRKAN_F32))
        return GRKAN_ERR_ALIGN;
    if (rows == 0)
        return GRKAN_OK;
    const norm::Variant v = norm::choose(D, io, weight_dtype, scale ? 1 : 0, residual != nullptr);
    norm::Args a = {};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.h = h;
    a.y = y;
    a.scale = scale;
    a.rows = rows;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.D = D;
    a.eps = eps;
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3((unsigned)norm::grid_of(v, rows, D, io, false)), dim3((unsigned)v.threads), args,
                        0, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    return GRKAN_OK;
}

extern "C" size_t grkan_rms_norm_bwd_workspace_bytes(int64_t rows, int32_t D, grkan_dtype_t io)
{
    if (norm::check(rows, D, io, GRKAN_F32) != GRKAN_OK)
        return 0;
    const norm::Variant v = norm::choose(D, io, GRKAN_F32, 2, false);
    const int64_t grid = norm::grid_of(v, rows, D, io, true);
    return (size_t)(grid > 0 ? grid : 1) * (size_t)D * sizeof(float);
}

extern "C" grkan_status_t grkan_rms_norm_bwd(const void *h, const void *dy, const void *dh, const void *weight, void *dx, void *dweight,
                                             void *workspace, size_t workspace_bytes, int64_t rows, int32_t D, int64_t h_stride,
                                             int64_t dy_stride, int64_t dh_stride, float eps, grkan_dtype_t io,
                                             grkan_dtype_t weight_dtype, void *hip_stream)
{
    const grkan_status_t bad = norm::check(rows, D, io, weight_dtype);
    if (bad != GRKAN_OK)
        return bad;
    if (!weight || !dweight || (rows > 0 && (!h || !dy || !dx)))
        return GRKAN_ERR_NULL;
    if (norm::misaligned(h, io) || norm::misaligned(dy, io) || norm::misaligned(dh, io) || norm::misaligned(dx, io) ||
        norm::misaligned(weight, weight_dtype) || norm::misaligned(dweight, weight_dtype))
        return GRKAN_ERR_ALIGN;
    const norm::Variant v = norm::choose(D, io, weight_dtype, 2, dh != nullptr);
    const int64_t grid = norm::grid_of(v, rows, D, io, true);
    if (!workspace || workspace_bytes < (size_t)grid * (size_t)D * sizeof(float) || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return GRKAN_ERR_WORKSPACE;
    hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
    norm::Args a = {};
    a.x = h;
    a.residual = dh;
    a.weight = weight;
    a.dy = dy;
    a.y = dx;
    a.partial = static_cast<float *>(workspace);
    a.rows = rows;
    a.x_stride = h_stride;
    a.residual_stride = dh_stride;
    a.dy_stride = dy_stride;
    a.D = D;
    a.eps = eps;
    if (grid > 0) {
        void *args[] = {&a};
        if (hipLaunchKernel(reinterpret_cast<const void *>(v.kernel), dim3((unsigned)grid), dim3((unsigned)v.threads), args, 0, stream) !=
            hipSuccess)
            return GRKAN_ERR_LAUNCH;
    }
    const dim3 blocks((unsigned)((D + 15) / 16));
    if (weight_dtype == GRKAN_F32)
        norm::columns_kernel<float><<<blocks, 1024, 0, stream>>>(a.partial, (int32_t)grid, D, static_cast<float *>(dweight));
    else if (weight_dtype == GRKAN_BF16)
        norm::columns_kernel<__bf16><<<blocks, 1024, 0, stream>>>(a.partial, (int32_t)grid, D, static_cast<__bf16 *>(dweight));
    else
        norm::columns_kernel<_Float16><<<blocks, 1024, 0, stream>>>(a.partial, (int32_t)grid, D, static_cast<_Float16 *>(dweight));
    return hipGetLastError() == hipSuccess ? GRKAN_OK : GRKAN_ERR_LAUNCH;
}
