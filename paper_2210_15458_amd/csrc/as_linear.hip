// Layers: products with bias, activation, residual and shaping in their epilogue.
#include <math.h>

#include <type_traits>

#include "as_shape.hpp"

namespace as {

// ---------------------------------------------------------------- epilogue

// tanh x = 1 - 2 / (1 + e^2x), by its series below 1/4, where that difference would cancel (its next term is 8e-9 there)
__device__ __forceinline__ float tanh_of(float x)
{
    const float q = x * x;
    const float s = x * (1.f + q * (-1.f / 3.f + q * (2.f / 15.f + q * (-17.f / 315.f + q * (62.f / 2835.f)))));
    const float e = __builtin_amdgcn_exp2f(2.88539008177792681472f * fabsf(x));
    const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + e);
    return fabsf(x) < 0.25f ? s : copysignf(t, x);
}

__device__ __forceinline__ float activate(float z, int act, float arg, float inv)
{
    switch (act) {
    case AS_ACT_RELU: return z < 0.f ? 0.f : z;                       // (NaN stays)
    case AS_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752440f));
    // z/2 (1 + tanh u) = z / (1 + e^-2u)
    case AS_ACT_GELU_TANH: {
        const float u = z * (0.79788456080286535588f + 0.79788456080286535588f * 0.044715f * z * z);
        return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.88539008177792681472f * u));
    }
    case AS_ACT_SILU: return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z));
    case AS_ACT_SOFTCAP: return arg * tanh_of(z * inv);
    default: return z;
    }
}

// Eight sums of one row, columns col .. col + 7 (col a multiple of 8 below n): everything behind the product, in fp32, with
// one rounding at the store.
template <class OutT>
__device__ __forceinline__ void finish8(const LinearArgs &a, int64_t row, int32_t col, float (&z)[8])
{
    const f32x4 b0 = *reinterpret_cast<const f32x4 *>(a.bias + col), b1 = *reinterpret_cast<const f32x4 *>(a.bias + col + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = activate(z[e] * a.scale + (e < 4 ? b0[e & 3] : b1[e & 3]), a.act, a.act_arg, a.act_inv);
    if (a.shaped && a.shape.finished && a.shape.finished[row]) return;
    const OutT *const add = (const OutT *)a.residual + row * a.ldr + col;
    OutT *const to = (OutT *)a.out + row * a.ldo + col;
    const int left = a.n - col;
    if (left >= 8) {
        if (a.residual) {
            Raw8<OutT> raw;
            float r[8];
            load_raw8(add, raw);
            widen8(raw, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] += r[e];
        }
        if (a.shaped) {
            const ShapeRow r = shape_row<false>(a.shape, row);
            Shape8 p;
            shape8_request(r, col, p);
            shape8_counts(r, col, p);
            shape8_apply(r, col, p, z);
        }
        store8(to, z);
    } else {
        const ShapeRow r = shape_row<false>(a.shape, row);           // (nothing in it where there is no shaping)
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) store1(to + e, shape_one(r, col + e, a.residual ? z[e] + widen(add[e]) : z[e]));
    }
}

// ---------------------------------------------------------------- any product

// 64 x 64 of the output a block, 32 k at a time through LDS, v_mfma_f32_16x16x4_f32: lane l holds k = l / 16 of row l % 16
// of either operand, and of the result column l % 16 and rows 4 (l / 16) .. + 3.
template <class T, class OutT>
__global__ __launch_bounds__(256) void linear_any(LinearArgs a, int32_t mtiles)
{
    constexpr int KS = 32, kStride = KS + 4, kOut = 64 + 4;
    __shared__ __attribute__((aligned(16))) float lds[2 * 64 * kStride > 64 * kOut ? 2 * 64 * kStride : 64 * kOut];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t m0 = (int64_t)(blockIdx.x % mtiles) * 64;
    const int32_t n0 = (int32_t)(blockIdx.x / mtiles) * 64;
    const T *x = (const T *)a.x, *W = (const T *)a.W;
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wm = wave >> 1, wn = wave & 1;
    for (int32_t k0 = 0; k0 < a.k; k0 += KS) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int u = tid + i * 256, r = u / KS, k = k0 + u % KS;          // rows 0..63 of x, 64..127 of W
            float v = 0.f;
            if (r < 64) {
                if (m0 + r < a.rows && k < a.k) v = widen(x[(m0 + r) * a.ldx + k]);
            } else if (n0 + r - 64 < a.n && k < a.k) {
                v = widen(W[(int64_t)(n0 + r - 64) * a.ldw + k]);
            }
            lds[r * kStride + u % KS] = v;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < KS; kk += 4) {
            float fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fa[i] = lds[(wm * 32 + i * 16 + (lane & 15)) * kStride + kk + (lane >> 4)];
                fb[i] = lds[(64 + wn * 32 + i * 16 + (lane & 15)) * kStride + kk + (lane >> 4)];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                lds[(wm * 32 + i * 16 + 4 * (lane >> 4) + v) * kOut + wn * 32 + j * 16 + (lane & 15)] = acc[i][j][v];
    __syncthreads();
    for (int u = tid; u < 64 * 8; u += 256) {
        const int r = u >> 3, c = (u & 7) * 8;
        if (m0 + r >= a.rows || n0 + c >= a.n) continue;
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = lds[r * kOut + c + e];
        finish8<OutT>(a, m0 + r, n0 + c, z);
    }
}

// ---------------------------------------------------------------- layer

// The layer's bias in fp32, zeros behind it up to a whole number of 256 columns (and everywhere, where it has none); and the
// weights in rows of kp, zeros behind k, where the caller's rows are not of that kind.
template <class T> __global__ __launch_bounds__(256) void layer_bias_kernel(const T *bias, float *out, int32_t n, int32_t padded)
{
    const int32_t i = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (i < padded) out[i] = bias && i < n ? widen(bias[i]) : 0.f;
}
__global__ __launch_bounds__(256) void layout_kernel(const uint16_t *in, int64_t ld, int64_t rows, int32_t k, uint16_t *out, int32_t kp)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / kp;
    const int32_t c = (int32_t)(i - row * kp);
    if (row < rows) out[i] = c < k ? in[row * ld + c] : 0;
}

as_status launch_layer_layout(const as_layer &l, const void *W, int64_t ldw, const void *bias)
{
    const int32_t padded = (l.n + 255) / 256 * 256;
    const dim3 grid((unsigned)(padded / 256));
    if (l.wdtype == AS_BF16)
        hipLaunchKernelGGL(layer_bias_kernel<uint16_t>, grid, dim3(256), 0, nullptr, (const uint16_t *)bias, l.bias, l.n, padded);
    else
        hipLaunchKernelGGL(layer_bias_kernel<float>, grid, dim3(256), 0, nullptr, (const float *)bias, l.bias, l.n, padded);
    AS_HIP_TRY(nullptr, hipGetLastError());
    if (l.own) {
        const int64_t blocks = ((int64_t)l.n * l.kp + 255) / 256;
        if (blocks > 0x7fffffffLL) return fail(nullptr, AS_ERR_UNSUPPORTED, "weights too large to lay out");
        hipLaunchKernelGGL(layout_kernel, dim3((unsigned)blocks), dim3(256), 0, nullptr, (const uint16_t *)W, ldw, (int64_t)l.n, l.k,
                           (uint16_t *)l.own, l.kp);
        AS_HIP_TRY(nullptr, hipGetLastError());
    }
    AS_HIP_TRY(nullptr, hipStreamSynchronize(nullptr));
    return AS_OK;
}

// ---------------------------------------------------------------- launch

size_t linear_workspace(const as_layer *l, const void *x, int64_t rows, int64_t ldx)
{
    return 0;
}

as_status launch_linear(as_ctx *ctx, const as_layer *l, LinearArgs a)
{
    const int64_t mtiles = (a.rows + 63) / 64, blocks = mtiles * ((a.n + 63) / 64);
    if (blocks > 0x7fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "product too large for one launch");
    const dim3 grid((unsigned)blocks);
    if (l->wdtype == AS_F32)
        launch(ctx, kKernelLogits, linear_any<float, float>, grid, dim3(256), 0, a, (int32_t)mtiles);
    else if (a.out_dtype == AS_BF16)
        launch(ctx, kKernelLogits, linear_any<uint16_t, uint16_t>, grid, dim3(256), 0, a, (int32_t)mtiles);
    else
        launch(ctx, kKernelLogits, linear_any<uint16_t, float>, grid, dim3(256), 0, a, (int32_t)mtiles);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

}  // namespace as
