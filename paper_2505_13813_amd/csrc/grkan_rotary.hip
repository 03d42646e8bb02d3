// Rotary positions with several axes on gfx950 (MI355X): pair j of a head's channels is turned by positions[token][axis[j]] *
// frequencies[j], for queries and keys in one launch; the backward pass is the inverse rotation.
//
// Bound by memory: every element is read and written once, and a pair takes six operations.  The angle's sine and cosine are
// another matter (some eighty operations with the reduction in 64 bits), and the same for all heads of a token.  So a workgroup has a
// run of tokens: its lanes first compute their sines and cosines into LDS, once each, and then stream the tokens' heads, which lie
// one behind the other, in vectors of up to 16 bytes.  (128 images of 196 tokens, 12 + 12 heads of 64 in bfloat16: 28.5 us = 5.4 TB/s, where
// a large copy reaches 5.5, in float32 59 us = 5.2; two videos of 14,720 tokens, 16 + 4 heads of 128: 55.5 us = 5.4 TB/s.)
#include <hip/hip_runtime.h>

#include "../../include/grkan_transformer.h"
#include "grkan_vector.h"

namespace grkan {
namespace rotary {

using namespace vec;

constexpr int kThreads = 256, kMostAngles = 4096;       // angles of a workgroup in LDS: 32 KB
constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1; // a launch has less than 2^32 threads

struct Tensor {
    const char *x;
    char *out;
    const char *positions;
    int64_t tokens, all_tokens; // of a batch entry, of all
    int64_t batch_stride, token_stride, head_stride, position_batch_stride, position_token_stride;
    int32_t heads, positions_dtype, per_block; // per_block: tokens of a workgroup
    uint32_t by_heads; // 2^32 / heads, rounded up (below: by chunks): quotients of small numbers by the high half of a product; 0: of one
};

struct Args {
    Tensor t[2];
    int64_t first_blocks; // of t[0]
    const double *frequencies;
    const int32_t *axis;
    int32_t pairs, axes, dim;
    uint32_t chunks, by_chunks; // items of 2 VP channels a head
    float sign; // of the angle
};

// VP pairs an item: 2 VP channels.
template <typename IO, int VP, bool INTERLEAVED> __global__ __launch_bounds__(kThreads) void rotary_kernel(const Args a)
{
    extern __shared__ __align__(16) float turned[]; // cos, sin of each token's pairs
    const bool second = (int64_t)blockIdx.x >= a.first_blocks;
    const Tensor &t = a.t[second];
    const int64_t token0 = ((int64_t)blockIdx.x - (second ? a.first_blocks : 0)) * t.per_block;
    const int64_t left = t.all_tokens - token0;
    const uint32_t tokens = (uint32_t)(left < t.per_block ? left : t.per_block);
    const uint32_t pairs = (uint32_t)a.pairs;

    for (uint32_t i = threadIdx.x; i < tokens * pairs; i += kThreads) {
        const uint32_t k = i / pairs, j = i - k * pairs;
        const int64_t token = token0 + k, b = token / t.tokens;
        int32_t ax = a.axis[j];
        ax = ax < 0 ? 0 : ax < a.axes ? ax : a.axes - 1;
        const int64_t at = b * t.position_batch_stride + (token - b * t.tokens) * t.position_token_stride + ax;
        const double position = t.positions_dtype == GRKAN_POSITIONS_I32   ? (double)reinterpret_cast<const int32_t *>(t.positions)[at]
                                : t.positions_dtype == GRKAN_POSITIONS_I64 ? (double)reinterpret_cast<const int64_t *>(t.positions)[at]
                                                                           : (double)reinterpret_cast<const float *>(t.positions)[at];
        // in turns, less the whole ones
        double turns = position * (a.frequencies[j] * 0.15915494309189533577);
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        turned[2 * i] = c;
        turned[2 * i + 1] = s * a.sign;
    }
    __syncthreads();

    // Items in turns of kAtOnce a lane, whose loads are all out before the first is used.
    constexpr int kAtOnce = 2;
    const uint32_t heads = (uint32_t)t.heads, rotated = pairs / VP, items = tokens * heads * a.chunks;
    IO *const out = reinterpret_cast<IO *>(t.out) + token0 * t.heads * a.dim;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += kThreads * kAtOnce) {
        typename Raw<IO, VP>::type first[kAtOnce], second[kAtOnce];
        uint32_t from[kAtOnce], to[kAtOnce], angle[kAtOnce]; // the vectors' channels; the first of the item's angles, or ~0: copied
        uint32_t line[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const uint32_t i = i0 + (uint32_t)u * kThreads;
            if (u > 0 && i >= items)
                continue;
            line[u] = a.by_chunks ? __umulhi(i, a.by_chunks) : i;
            const uint32_t c = i - line[u] * a.chunks, k = t.by_heads ? __umulhi(line[u], t.by_heads) : line[u], h = line[u] - k * heads;
            const int64_t token = token0 + k, b = t.tokens == t.all_tokens ? 0 : token / t.tokens;
            const IO *const x = reinterpret_cast<const IO *>(t.x) + b * t.batch_stride + (token - b * t.tokens) * t.token_stride + h * t.head_stride;
            const bool turns = c < rotated;
            from[u] = turns && !INTERLEAVED ? c * VP : c * 2 * VP;
            to[u] = turns && !INTERLEAVED ? pairs + from[u] : from[u] + VP;
            angle[u] = turns ? k * pairs + c * VP : ~0u;
            first[u] = load<IO, VP>(x + from[u]);
            second[u] = load<IO, VP>(x + to[u]);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (u > 0 && i0 + (uint32_t)u * kThreads >= items)
                continue;
            float f[2 * VP], lo[VP], hi[VP];
            widen<IO, VP>(first[u], lo);
            widen<IO, VP>(second[u], hi);
#pragma unroll
            for (int e = 0; e < VP; ++e) {
                f[e] = lo[e];
                f[VP + e] = hi[e];
            }
            if (angle[u] != ~0u) {
                const float *const cs = turned + 2 * angle[u];
#pragma unroll
                for (int j = 0; j < VP; ++j) {
                    const int ia = INTERLEAVED ? 2 * j : j, ib = INTERLEAVED ? 2 * j + 1 : VP + j;
                    const float p = f[ia], q = f[ib], co = cs[2 * j], si = cs[2 * j + 1];
                    f[ia] = p * co - q * si;
                    f[ib] = p * si + q * co;
                }
            }
#pragma unroll
            for (int e = 0; e < VP; ++e) {
                lo[e] = f[e];
                hi[e] = f[VP + e];
            }
            IO *const o = out + (int64_t)line[u] * a.dim;
            store<IO, VP>(o + from[u], narrow<IO, VP>(lo));
            store<IO, VP>(o + to[u], narrow<IO, VP>(hi));
        }
    }
}

typedef void (*Kernel)(Args);
template <typename IO, int VP> static Kernel pick(bool interleaved)
{
    return interleaved ? rotary_kernel<IO, VP, true> : rotary_kernel<IO, VP, false>;
}

static Kernel choose(grkan_dtype_t io, int vp, bool interleaved)
{
    if (io == GRKAN_F32)
        return vp == 4 ? pick<float, 4>(interleaved) : vp == 2 ? pick<float, 2>(interleaved) : pick<float, 1>(interleaved);
    if (io == GRKAN_BF16)
        return vp == 8   ? pick<__bf16, 8>(interleaved)
               : vp == 4 ? pick<__bf16, 4>(interleaved)
               : vp == 2 ? pick<__bf16, 2>(interleaved)
                         : pick<__bf16, 1>(interleaved);
    return vp == 8   ? pick<_Float16, 8>(interleaved)
           : vp == 4 ? pick<_Float16, 4>(interleaved)
           : vp == 2 ? pick<_Float16, 2>(interleaved)
                     : pick<_Float16, 1>(interleaved);
}

} // namespace rotary
} // namespace grkan

using namespace grkan;

extern "C" grkan_status_t grkan_rotary(const grkan_rotary_t *tensors, int32_t count, const double *frequencies, const int32_t *axis,
                                       int32_t pairs, int32_t axes, int32_t dim, int32_t interleaved, int32_t inverse, grkan_dtype_t io,
                                       void *hip_stream)
{
    if (!tensors)
        return GRKAN_ERR_NULL;
    if (count < 1 || count > 2 || pairs < 0 || axes < 1 || dim < 1 || pairs > dim / 2)
        return GRKAN_ERR_SHAPE;
    if (io != GRKAN_F32 && io != GRKAN_BF16 && io != GRKAN_F16)
        return GRKAN_ERR_DTYPE;
    if (dim % 2 != 0 || dim > 4096)
        return GRKAN_ERR_UNSUPPORTED;
    if (pairs > 0 && (!frequencies || !axis))
        return GRKAN_ERR_NULL;
    const uintptr_t element = io == GRKAN_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(frequencies) % 8 != 0 || reinterpret_cast<uintptr_t>(axis) % 4 != 0)
        return GRKAN_ERR_ALIGN;
    // the longest vector that both the turned and the other channels are whole numbers of
    int vp = 16 / (int)element;
    while (pairs % vp != 0 || dim / 2 % vp != 0)
        vp /= 2;
    rotary::Args a = {};
    int64_t blocks = 0;
    int32_t most_tokens = 1;
    for (int i = 0; i < count; ++i) {
        const grkan_rotary_t &t = tensors[i];
        if (t.batch < 0 || t.tokens < 0 || t.heads < 1)
            return GRKAN_ERR_SHAPE;
        if (t.positions_dtype != GRKAN_POSITIONS_I32 && t.positions_dtype != GRKAN_POSITIONS_I64 && t.positions_dtype != GRKAN_POSITIONS_F32)
            return GRKAN_ERR_DTYPE;
        if (t.heads > 65536 || t.batch > INT32_MAX || t.tokens > INT32_MAX)
            return GRKAN_ERR_UNSUPPORTED;
        const int64_t all = t.batch * t.tokens;
        if (all > 0 && (!t.x || !t.out || (pairs > 0 && !t.positions)))
            return GRKAN_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.out)) % element != 0 ||
            reinterpret_cast<uintptr_t>(t.positions) % (t.positions_dtype == GRKAN_POSITIONS_I64 ? 8 : 4) != 0)
            return GRKAN_ERR_ALIGN;
        // n / d = high half of n ceil(2^32 / d) where n d < 2^32
        const uint64_t chunks = (uint64_t)(dim / (2 * vp)), one = (uint64_t)t.heads * chunks;
        // Two items a lane, all out at once, where there are tokens enough for two workgroups on
        // every compute unit (us with 1 / 2 / 4 / 8 items: 128 images of 196 tokens, 12 + 12 heads
        // of 64, 29 / 28 / 31 / 34; two videos of 14,720, 16 + 4 heads of 128, 57 / 55 / 60 / 68).
        int64_t per = 2 * rotary::kThreads / (int64_t)one;
        per = per < all / 512 ? per : all / 512;
        per = per < rotary::kMostAngles / (pairs > 0 ? pairs : 1) ? per : rotary::kMostAngles / (pairs > 0 ? pairs : 1);
        per = per > 1 ? per : 1;
        if ((uint64_t)per * one * (chunks > (uint64_t)t.heads ? chunks : (uint64_t)t.heads) >> 32)
            return GRKAN_ERR_UNSUPPORTED;
        rotary::Tensor &to = a.t[i];
        to.x = static_cast<const char *>(t.x);
        to.out = static_cast<char *>(t.out);
        to.positions = static_cast<const char *>(t.positions);
        to.tokens = t.tokens > 0 ? t.tokens : 1;
        to.all_tokens = all;
        to.batch_stride = t.batch_stride;
        to.token_stride = t.token_stride;
        to.head_stride = t.head_stride;
        to.position_batch_stride = t.position_batch_stride;
        to.position_token_stride = t.position_token_stride;
        to.heads = t.heads;
        to.positions_dtype = t.positions_dtype;
        to.per_block = (int32_t)per;
        to.by_heads = t.heads > 1 ? (uint32_t)((((uint64_t)1 << 32) + (uint64_t)t.heads - 1) / (uint64_t)t.heads) : 0;
        most_tokens = per > most_tokens ? (int32_t)per : most_tokens;
        blocks += (all + per - 1) / per;
        if (i == 0)
            a.first_blocks = blocks;
    }
    if (blocks > rotary::kMostBlocks)
        return GRKAN_ERR_UNSUPPORTED;
    if (blocks == 0)
        return GRKAN_OK;
    a.frequencies = frequencies;
    a.axis = axis;
    a.pairs = pairs;
    a.axes = axes;
    a.dim = dim;
    a.chunks = (uint32_t)(dim / (2 * vp));
    a.by_chunks = a.chunks > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.chunks - 1) / a.chunks) : 0;
    a.sign = inverse ? -1.0f : 1.0f;
    void *args[] = {&a};
    if (hipLaunchKernel(reinterpret_cast<const void *>(rotary::choose(io, vp, interleaved != 0)), dim3((unsigned)blocks), dim3(rotary::kThreads),
                        args, (size_t)most_tokens * (size_t)pairs * 8, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return GRKAN_ERR_LAUNCH;
    return GRKAN_OK;
}
