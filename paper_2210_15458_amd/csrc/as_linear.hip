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

// ---------------------------------------------------------------- tiles (bf16)

// One block, four waves, a tile of TM x TN outputs.  The waves stand WM x WN x KG: KG groups share the tile's sum, group g
// taking every KG-th of the K stages of 64, and add what they have in the epilogue, in the order of g.  So a product with few
// tiles still has four waves on each, with that many more loads on their way, and no second launch to join them.
//
// Operands go global -> LDS directly (lane l's 16 bytes land at base + 16 l), 128 bytes of 8 rows a request, into a ring of
// RING steps; LDS rows are 128 bytes with 16-byte piece c of row r at c ^ ((r >> 1) & 7), so that neither the fragment
// reads nor the loads meet a bank twice.  Rows past either end repeat the last one and are not stored.
// v_mfma_f32_32x32x16_bf16 with W as its first operand: register v of lane l is column 8 (v / 4) + 4 (l / 32) + v % 4 and
// row l % 32 of the 32 x 32, so that a lane holds runs of four consecutive outputs.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_void;
constexpr int kStageK = 64;

// the fragments of two K slices: all reads and their wait in one piece of text, so that nothing comes between a read in
// flight and its register
template <int FM, int FN> struct Frags {
    bf16x8 w[2][FN], x[2][FM];
};
template <int FM, int FN>
__device__ __forceinline__ void read_frags(Frags<FM, FN> &f, uint32_t w0, uint32_t x0, uint32_t w1, uint32_t x1)
{
    if constexpr (FM == 1 && FN == 1) {
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(f.w[0][0]), "=&v"(f.x[0][0]), "=&v"(f.w[1][0]), "=&v"(f.x[1][0])
                     : "v"(w0), "v"(x0), "v"(w1), "v"(x1)
                     : "memory");
    } else if constexpr (FM == 2 && FN == 1) {
        asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\tds_read_b128 %2, %7 offset:4096\n\t"
                     "ds_read_b128 %3, %8\n\tds_read_b128 %4, %9\n\tds_read_b128 %5, %9 offset:4096\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(f.w[0][0]), "=&v"(f.x[0][0]), "=&v"(f.x[0][1]), "=&v"(f.w[1][0]), "=&v"(f.x[1][0]), "=&v"(f.x[1][1])
                     : "v"(w0), "v"(x0), "v"(w1), "v"(x1)
                     : "memory");
    } else {
        static_assert(FM == 2 && FN == 2, "the forms that there are");
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:4096\n\t"
                     "ds_read_b128 %2, %9\n\tds_read_b128 %3, %9 offset:4096\n\t"
                     "ds_read_b128 %4, %10\n\tds_read_b128 %5, %10 offset:4096\n\t"
                     "ds_read_b128 %6, %11\n\tds_read_b128 %7, %11 offset:4096\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(f.w[0][0]), "=&v"(f.w[0][1]), "=&v"(f.x[0][0]), "=&v"(f.x[0][1]), "=&v"(f.w[1][0]), "=&v"(f.w[1][1]),
                       "=&v"(f.x[1][0]), "=&v"(f.x[1][1])
                     : "v"(w0), "v"(x0), "v"(w1), "v"(x1)
                     : "memory");
    }
}

template <class OutT, int WM, int WN, int KG, int FM, int FN, int RING>
__global__ __launch_bounds__(256) void linear_tile(LinearArgs a, uint32_t mtiles, uint32_t ntiles)
{
    static_assert(WM * WN * KG == 4 && (RING & (RING - 1)) == 0, "four waves; a ring of a power of two");
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32, kRows = TM + TN;
    constexpr int kPart = kRows * 128, kStep = KG * kPart;            // bytes of a group's stage, of a step
    constexpr int kPer = kRows / 32;                                  // requests of a wave for a group's stage
    constexpr int kStride = TN + 4;                                   // floats of a staged row of sums
    constexpr int kOut = KG * TM * kStride * 4;
    constexpr int kLds = RING * kStep > kOut ? RING * kStep : kOut;
    static_assert(kLds <= 160 * 1024 && (RING - 2) * kPer * KG < 64, "LDS, and what the wait can count");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kLds];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
    // blocks of one column tile follow each other eight apart, on one XCD: its rows of W come through that L2 once
    const uint32_t bid = blockIdx.x, eight = bid / (8 * mtiles), in = bid % (8 * mtiles);
    const uint32_t across = ntiles - eight * 8 < 8 ? ntiles - eight * 8 : 8;
    const int32_t n0 = (int32_t)((eight * 8 + in % across) * TN);
    const int64_t m0 = (int64_t)(in / across) * TM;

    // a wave's requests: rows i * 32 + wave * 8 + lane / 8 of the part, W's first
    const int rl = wave * 8 + (lane >> 3);
    const uint32_t piece = (uint32_t)(((lane & 7) ^ ((rl >> 1) & 7)) << 4);
    const unsigned char *from[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = i * 32 + rl;
        if (i * 32 < TN) {
            const int32_t n = n0 + r < a.n ? n0 + r : a.n - 1;
            from[i] = (const unsigned char *)a.W + (int64_t)n * a.ldw * 2 + piece;
        } else {
            const int64_t m = m0 + r - TN < a.rows ? m0 + r - TN : a.rows - 1;
            from[i] = (const unsigned char *)a.x + m * a.ldx * 2 + piece;
        }
    }
    const int stages = a.k / kStageK, steps = (stages + KG - 1) / KG;
    auto request = [&](int step) __attribute__((always_inline)) {
        unsigned char *const slot = smem + (step & (RING - 1)) * kStep + wave * 1024;
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            const int st = step * KG + g < stages ? step * KG + g : stages - 1;   // (past the end: loaded, not used)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                __builtin_amdgcn_global_load_lds((glb_void *)(from[i] + (int64_t)st * (kStageK * 2)),
                                                 (lds_void *)(slot + g * kPart + i * 4096), 16, 0, 0);
        }
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int frow = lane & 31;
    const uint32_t sw = (uint32_t)(((lane >> 5) ^ ((frow >> 1) & 7)) << 4);
    const uint32_t fw = lds0 + kg * kPart + (uint32_t)(wn * FN * 32 + frow) * 128 + sw;
    const uint32_t fx = lds0 + kg * kPart + (uint32_t)(TN + wm * FM * 32 + frow) * 128 + sw;
    for (int s = 0; s < RING - 1 && s < steps; ++s) request(s);
    for (int s = 0; s < steps; ++s) {
        // step s has landed; up to RING - 2 more stay on their way
        const int behind = steps - 1 - s;
        if (behind >= RING - 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 2) * kPer * KG) : "memory");
        else if (RING > 3 && behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPer * KG) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (every wave has left step s - 1, whose slot this is)
        if (s + RING - 1 < steps) request(s + RING - 1);
        if (KG > 1 && s * KG + kg >= stages) continue;
        const uint32_t so = (uint32_t)(s & (RING - 1)) * kStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Frags<FM, FN> f;
            read_frags<FM, FN>(f, (fw + so) ^ (uint32_t)(h * 64), (fx + so) ^ (uint32_t)(h * 64), (fw + so) ^ (uint32_t)(h * 64 + 32),
                               (fx + so) ^ (uint32_t)(h * 64 + 32));
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.w[q][j], f.x[q][i], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();                                                  // the ring gives way to the sums
    float *const sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(sums + (kg * TM + (wm * FM + i) * 32 + (lane & 31)) * kStride + (wn * FN + j) * 32 + 8 * q +
                                           4 * (lane >> 5)) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    for (int u = tid; u < TM * TN / 8; u += 256) {
        const int r = u / (TN / 8), c = u % (TN / 8) * 8;
        if (m0 + r >= a.rows || n0 + c >= a.n) continue;
        float z[8];
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(sums + (g * TM + r) * kStride + c),
                        hi = *reinterpret_cast<const f32x4 *>(sums + (g * TM + r) * kStride + c + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (g == 0 ? 0.f : z[e]) + (e < 4 ? lo[e & 3] : hi[e & 3]);
        }
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

// Whether rows of x can be read as they are: whole pieces of 16 bytes, whole stages of K.
static bool x_as_it_is(const as_layer *l, const void *x, int64_t ldx)
{
    return l->kp == l->k && ldx % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
}

size_t linear_workspace(const as_layer *l, const void *x, int64_t rows, int64_t ldx)
{
    return l->wdtype == AS_BF16 && !x_as_it_is(l, x, ldx) ? (size_t)rows * l->kp * 2 : 0;
}

template <class OutT, int WM, int WN, int KG, int FM, int FN, int RING> static as_status launch_tile(as_ctx *ctx, const LinearArgs &a)
{
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32;
    const int64_t mtiles = (a.rows + TM - 1) / TM, ntiles = (a.n + TN - 1) / TN;
    if (mtiles * ntiles > 0x7fffffffLL || mtiles > 0x0fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "product too large for one launch");
    launch(ctx, kKernelLogits, linear_tile<OutT, WM, WN, KG, FM, FN, RING>, dim3((unsigned)(mtiles * ntiles)), dim3(256), 0, a,
           (uint32_t)mtiles, (uint32_t)ntiles);
    return AS_OK;
}

template <class OutT> static as_status launch_bf16(as_ctx *ctx, const LinearArgs &a)
{
    switch (ctx->linear_shape) {
    case 1: return launch_tile<OutT, 1, 1, 4, 1, 1, 4>(ctx, a);      // 32 x 32, four groups
    case 2: return launch_tile<OutT, 1, 2, 2, 1, 1, 4>(ctx, a);      // 32 x 64, two groups
    case 3: return launch_tile<OutT, 1, 4, 1, 1, 1, 4>(ctx, a);      // 32 x 128
    case 4: return launch_tile<OutT, 1, 4, 1, 2, 1, 4>(ctx, a);      // 64 x 128
    case 5: return launch_tile<OutT, 2, 2, 1, 2, 2, 4>(ctx, a);      // 128 x 128
    case 6: return launch_tile<OutT, 1, 1, 4, 2, 2, 2>(ctx, a);      // 64 x 64, four groups
    case 7: return launch_tile<OutT, 1, 2, 2, 2, 1, 4>(ctx, a);      // 64 x 64, two groups
    case 8: return launch_tile<OutT, 2, 2, 1, 1, 1, 4>(ctx, a);      // 64 x 64
    }
    return launch_tile<OutT, 1, 4, 1, 1, 1, 4>(ctx, a);
}

as_status launch_linear(as_ctx *ctx, const as_layer *l, LinearArgs a)
{
    as_status st = AS_OK;
    if (l->wdtype == AS_F32) {
        const int64_t mtiles = (a.rows + 63) / 64, blocks = mtiles * ((a.n + 63) / 64);
        if (blocks > 0x7fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "product too large for one launch");
        launch(ctx, kKernelLogits, linear_any<float, float>, dim3((unsigned)blocks), dim3(256), 0, a, (int32_t)mtiles);
    } else {
        if (!x_as_it_is(l, a.x, a.ldx)) {
            const int64_t blocks = (a.rows * l->kp + 255) / 256;
            if (blocks > 0x7fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "x too large to lay out");
            hipLaunchKernelGGL(layout_kernel, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, (const uint16_t *)a.x, a.ldx, a.rows,
                               l->k, (uint16_t *)ctx->linear_x.ptr, l->kp);
            a.x = ctx->linear_x.ptr;
            a.ldx = l->kp;
        }
        a.k = l->kp;
        st = a.out_dtype == AS_BF16 ? launch_bf16<uint16_t>(ctx, a) : launch_bf16<float>(ctx, a);
    }
    if (st != AS_OK) return st;
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

}  // namespace as
