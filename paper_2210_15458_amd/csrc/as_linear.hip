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

// The same in fewer steps: (1 - t) / (1 + t), t = e^-2|x|, whose difference is 2^-23 / 2|x| off, and two terms of the series
// below 1/32: at most 2e-6 off, a thousandth of the rounding to bf16 that follows.
__device__ __forceinline__ float tanh_for_bf16(float x)
{
    const float t = __builtin_amdgcn_exp2f(-2.88539008177792681472f * fabsf(x));
    const float y = copysignf((1.f - t) * __builtin_amdgcn_rcpf(1.f + t), x);
    return fabsf(x) < 0.03125f ? fmaf(x * (-1.f / 3.f), x * x, x) : y;
}

// z/2 (1 + erf(z / sqrt 2)) = z h or z (1 - h) with h = erfc(|z| / sqrt 2) / 2 = t P(t) e^(-z^2 / 2), t = 1 / (1 + p |z| / sqrt 2): no
// cancellation in the lower tail.  For outputs rounded to bf16 P is Abramowitz and Stegun 7.1.26, five terms, 7.5e-8 off at most (of
// h itself: 5e-4 at z = -4).  For fp32 outputs nine terms with p = 0.37, fitted by reweighted least squares to the smallest relative error
// over |z| < 13, 1.7e-8: what remains is the roundings', 4e-7 of the result at -1, 1.4e-6 at -5, where the argument of e is rounded.
template <class OutT> __device__ __forceinline__ float gelu_of(float z)
{
    constexpr bool SHORT = sizeof(OutT) == 2;
    const float t = __builtin_amdgcn_rcpf(fmaf((SHORT ? 0.3275911f : 0.37f) * 0.70710678118654752440f, fabsf(z), 1.f));
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170368f * (z * z));
    float c;
    if constexpr (SHORT) {
        c = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, -0.5f * 1.453152027f), 0.5f * 1.421413741f),
                             -0.5f * 0.284496736f), 0.5f * 0.254829592f);
    } else {
        constexpr float P[9] = {0.10440687f, 0.10371493f, 0.10312697f, 0.053260326f, 0.15540063f,
                                -0.14265543f, 0.2434205f, -0.15163632f, 0.030961514f};
        c = P[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) c = fmaf(t, c, P[i]);
        c *= t;
    }
    const float h = c * e;
    return z * (z > 0.f ? 1.f - h : h);
}

// The activation of N sums: the choice once, outside.
template <class OutT, int N, class V> __device__ __forceinline__ void activate(V &z, int act, float arg, float inv)
{
    switch (act) {
    case AS_ACT_RELU:
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = z[e] < 0.f ? 0.f : z[e];   // (NaN stays)
        break;
    case AS_ACT_GELU:
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = gelu_of<OutT>(z[e]);
        break;
    case AS_ACT_GELU_TANH:                                            // z/2 (1 + tanh u) = z / (1 + e^-2u)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float u = z[e] * (0.79788456080286535588f + 0.79788456080286535588f * 0.044715f * z[e] * z[e]);
            z[e] = z[e] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.88539008177792681472f * u));
        }
        break;
    case AS_ACT_SILU:
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = z[e] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z[e]));
        break;
    case AS_ACT_SOFTCAP:
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = arg * (sizeof(OutT) == 2 ? tanh_for_bf16(z[e] * inv) : tanh_of(z[e] * inv));
        break;
    }
}

// Eight outputs of one row, columns col .. col + 7 (col a multiple of 8 below n): what follows the activation, in fp32, with
// one rounding at the store.
template <class OutT, bool RESIDUAL = true, bool SHAPED = true>
__device__ __forceinline__ void finish8(const LinearArgs &a, int64_t row, int32_t col, float (&z)[8])
{
    const bool shaped = SHAPED && a.shaped, more = RESIDUAL && a.residual;
    if (shaped && a.shape.finished && a.shape.finished[row]) return;
    const OutT *const add = (const OutT *)a.residual + row * a.ldr + col;
    OutT *const to = (OutT *)a.out + row * a.ldo + col;
    const int left = a.n - col;
    if (left >= 8) {
        if (more) {
            Raw8<OutT> raw;
            float r[8];
            load_raw8(add, raw);
            widen8(raw, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] += r[e];
        }
        if (shaped) {
            const ShapeRow r = shape_row<false>(a.shape, row);
            Shape8 p;
            shape8_request(r, col, p);
            shape8_counts(r, col, p);
            shape8_apply(r, col, p, z);
        }
        store8(to, z);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            if (e >= left) continue;
            float y = more ? z[e] + widen(add[e]) : z[e];
            if (shaped) y = shape_one(shape_row<false>(a.shape, row), col + e, y);
            store1(to + e, y);
        }
    }
}

// The same from the sums.
template <class OutT>
__device__ __forceinline__ void finish8_sums(const LinearArgs &a, int64_t row, int32_t col, float (&z)[8])
{
    const f32x4 b0 = *reinterpret_cast<const f32x4 *>(a.bias + col), b1 = *reinterpret_cast<const f32x4 *>(a.bias + col + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = fmaf(z[e], a.scale, e < 4 ? b0[e & 3] : b1[e & 3]);
    activate<OutT, 8>(z, a.act, a.act_arg, a.act_inv);
    finish8<OutT>(a, row, col, z);
}

// What a thread finishes, eight columns of a row, whose own loads go out in two rounds: what the row and the columns say, ahead of
// the products, and what that points to, in the few-rows form between them, in the tiles behind the last.
template <class OutT> struct Unit {
    int64_t row;
    int32_t col;
    bool whole;                               // all eight inside
    Raw8<OutT> add;
    ShapeRow r;
    Shape8 p;

    __device__ __forceinline__ void first(const LinearArgs &a)
    {
        whole = row < a.rows && col + 8 <= a.n;
        if (!whole) return;
        if (a.residual) load_raw8((const OutT *)a.residual + row * a.ldr + col, add);
        if (a.shaped) {
            r = shape_row<false>(a.shape, row);
            if (r.seen) p.seen = r.seen[col >> 5];
        }
    }
    __device__ __forceinline__ void second(const LinearArgs &a)
    {
        if (!whole || !a.shaped) return;
        if (r.mask) p.mask = r.mask[col >> 5];
        if (r.bias) {
            p.bias[0] = *reinterpret_cast<const f32x4_any *>(r.bias + col);
            p.bias[1] = *reinterpret_cast<const f32x4_any *>(r.bias + col + 4);
        }
        shape8_counts(r, col, p);
    }
    __device__ __forceinline__ void finish(const LinearArgs &a, const f32x4 (&bias)[2], float (&z)[8])
    {
        if (row >= a.rows || col >= a.n) return;
        if (!whole) return finish8_sums<OutT>(a, row, col, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = fmaf(z[e], a.scale, bias[e >> 2][e & 3]);
        activate<OutT, 8>(z, a.act, a.act_arg, a.act_inv);
        if (a.residual) {
            float y[8];
            widen8(add, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] += y[e];
        }
        if (a.shaped) {
            if (a.shape.finished && a.shape.finished[row]) return;
            shape8_apply(r, col, p, z);
        }
        store8((OutT *)a.out + row * a.ldo + col, z);
    }
};

// What 256 threads finish of a tile of TM x TN: each always the same eight columns, of rows 256 / kAcross apart; two of them have
// their first loads out ahead of the products.  The sums lie in LDS, KG shares of TM rows, kStride floats apart, added in order.
template <class OutT, int TM, int TN, int KG> struct TileEnd {
    static constexpr int kAcross = TN / 8, kUnits = TM * kAcross > 256 ? TM * kAcross / 256 : 1, kAhead = kUnits < 2 ? 1 : 2;
    static constexpr int kStride = TN + 4, kBytes = KG * TM * kStride * 4;
    Unit<OutT> unit[kAhead];
    f32x4 bias[2];

    __device__ __forceinline__ void first(const LinearArgs &a, int64_t m0, int32_t n0)
    {
        const int tid = threadIdx.x;
        bias[0] = bias[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = u * (256 / kAcross) + tid / kAcross;
            unit[u].row = r < TM ? m0 + r : a.rows;
            unit[u].col = n0 + tid % kAcross * 8;
            unit[u].first(a);
        }
        if (unit[0].col < a.n) {
            bias[0] = *reinterpret_cast<const f32x4 *>(a.bias + unit[0].col);
            bias[1] = *reinterpret_cast<const f32x4 *>(a.bias + unit[0].col + 4);
        }
    }
    __device__ __forceinline__ void second(const LinearArgs &a)
    {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) unit[u].second(a);
    }
    __device__ __forceinline__ void finish(const LinearArgs &a, const float *sums)
    {
        const int tid = threadIdx.x;
        for (int u0 = 0; u0 < kUnits; u0 += kAhead) {
            if (u0 > 0) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    unit[u].row += kAhead * (256 / kAcross);
                    unit[u].first(a);
                }
                second(a);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int r = (u0 + u) * (256 / kAcross) + tid / kAcross;
                if (TM * kAcross < 256 && r >= TM) continue;
                float z[8];
#pragma unroll
                for (int g = 0; g < KG; ++g) {
                    const float *const at = sums + (g * TM + r) * kStride + tid % kAcross * 8;
                    const f32x4 lo = *reinterpret_cast<const f32x4 *>(at), hi = *reinterpret_cast<const f32x4 *>(at + 4);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = (g == 0 ? 0.f : z[e]) + (e < 4 ? lo[e & 3] : hi[e & 3]);
                }
                unit[u].finish(a, bias, z);
            }
        }
    }
};

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
// Bound by the round trips of a step (requests, barrier, fragments, products: some 500 cycles of 64 x 64 against 128 of products), which
// is why two to five blocks stand on a compute unit where there are tiles for them, and by the launch: 1024 x 512 x 2048 7.6 us (0.28
// PFLOP/s), 1024 x 2048 x 512 9.7, an empty sum of the size 2.7.  More stages ahead changed nothing (a ring of 6 for 4: 10.6 for 10.1).
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
    static_assert(WM * WN * KG == 4 && RING >= 2, "four waves; a slot to work on and one to fill");
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32, kRows = TM + TN;
    constexpr int kPart = kRows * 128, kStep = KG * kPart;            // bytes of a group's stage, of a step
    constexpr int kPer = kRows / 32;                                  // requests of a wave for a group's stage
    constexpr int kOut = TileEnd<OutT, TM, TN, KG>::kBytes;
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
    int fill = 0;                                                     // the slot of the next step to request
    auto request = [&](int step) __attribute__((always_inline)) {
        unsigned char *const slot = smem + fill * kStep + wave * 1024;
        fill = fill == RING - 1 ? 0 : fill + 1;
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
    TileEnd<OutT, TM, TN, KG> end;
    end.first(a, m0, n0);
    for (int s = 0; s < RING - 1 && s < steps; ++s) request(s);
    for (int s = 0, slot_of = 0; s < steps; ++s, slot_of = slot_of == RING - 1 ? 0 : slot_of + 1) {
        // step s has landed; up to RING - 2 more stay on their way
        const int behind = steps - 1 - s;
        if (behind >= RING - 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 2) * kPer * KG) : "memory");
        else if (RING > 6 && behind >= 4) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * kPer * KG) : "memory");
        else if (RING > 4 && behind >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kPer * KG) : "memory");
        else if (RING > 3 && behind >= 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPer * KG) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (every wave has left step s - 1, whose slot is filled: at once where nothing else is on its way, and where something is
        // behind the first products, which then need not wait for the requests to be taken)
        const bool more = s + RING - 1 < steps, idle = KG > 1 && s * KG + kg >= stages;
        if (more && (RING == 2 || idle)) request(s + RING - 1);
        if (idle) continue;
        const uint32_t so = (uint32_t)slot_of * kStep;
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
            if (RING > 2 && h == 0 && more) request(s + RING - 1);
        }
    }
    end.second(a);
    __syncthreads();                                                  // the ring gives way to the sums
    float *const sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(sums + (kg * TM + (wm * FM + i) * 32 + (lane & 31)) * end.kStride + (wn * FN + j) * 32 + 8 * q +
                                           4 * (lane >> 5)) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    end.finish(a, sums);
}

// ---------------------------------------------------------------- few rows (bf16)

// Up to 16 rows: a pass over W, each of whose elements one wave needs once, so that LDS would be a detour.  A wave takes 16 columns
// (v_mfma_f32_16x16x32_bf16, W first: lane l has 8 k from 8 (l / 16) on of row l % 16, and of the result row l % 16, columns
// 4 (l / 16) .. + 3) and one of KW shares of the sum, with U stages of 64 k, whole lines, on their way at once; the shares meet in
// LDS, in order.  WAVES / KW column groups a block.  Bound by one round trip to memory beside the launch where W is small (1 x 512 x
// 2048 3.0 us, an empty launch 2.2), by the memory where it is large (1 x 4096 x 4096 8.1 us, 4.1 TB/s; 1 x 1024 x 256000 79, 6.7).
template <class OutT, int WAVES, int KW, int U>
__global__ __launch_bounds__(WAVES * kWave) void linear_few(LinearArgs a)
{
    constexpr int WN = WAVES / KW, kStride = WN * 16 + 4, kUnits = 16 * WN * 2;
    static_assert(kUnits <= WAVES * kWave, "a unit a thread");
    __shared__ __attribute__((aligned(16))) float sums[KW * 16 * kStride];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / WN, wn = wave % WN, l = lane & 15, quarter = lane >> 4;
    const int32_t n0 = (int32_t)blockIdx.x * (WN * 16), mine = n0 + wn * 16 + l;
    const unsigned char *const w = (const unsigned char *)a.W + (int64_t)(mine < a.n ? mine : a.n - 1) * a.ldw * 2 + quarter * 16;
    const unsigned char *const x = (const unsigned char *)a.x + (l < a.rows ? l : a.rows - 1) * a.ldx * 2 + quarter * 16;
    const int stages = a.k / kStageK, from = stages * kg / KW, to = stages * (kg + 1) / KW;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    bf16x8 fw[U][2], fx[U][2];
    auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u >= to) break;
            const int64_t at = (int64_t)(s0 + u) * (kStageK * 2);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fw[u][h] = *reinterpret_cast<const bf16x8 *>(w + at + h * 64);
                fx[u][h] = *reinterpret_cast<const bf16x8 *>(x + at + h * 64);
            }
        }
    };
    auto multiply = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u >= to) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[u][h], fx[u][h], acc, 0, 0, 0);
        }
    };
    Unit<OutT> unit;
    unit.row = tid < kUnits ? tid / (WN * 2) : a.rows;
    unit.col = n0 + tid % (WN * 2) * 8;
    f32x4 bias[2] = {};
    if (from < to) load(from);
    unit.first(a);
    if (unit.col < a.n) {
        bias[0] = *reinterpret_cast<const f32x4 *>(a.bias + unit.col);
        bias[1] = *reinterpret_cast<const f32x4 *>(a.bias + unit.col + 4);
    }
    if (from < to) multiply(from);
    unit.second(a);
    for (int s0 = from + U; s0 < to; s0 += U) {
        load(s0);
        multiply(s0);
    }
    *reinterpret_cast<f32x4 *>(sums + (kg * 16 + l) * kStride + wn * 16 + quarter * 4) = acc;
    __syncthreads();
    if (tid >= kUnits) return;
    float z[8];
#pragma unroll
    for (int g = 0; g < KW; ++g) {
        const float *const at = sums + (g * 16 + tid / (WN * 2)) * kStride + tid % (WN * 2) * 8;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(at), hi = *reinterpret_cast<const f32x4 *>(at + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (g == 0 ? 0.f : z[e]) + (e < 4 ? lo[e & 3] : hi[e & 3]);
    }
    unit.finish(a, bias, z);
}

// ---------------------------------------------------------------- large products (bf16)

// A block of 8 waves (4 x 2, each 64 x 128 of 256 x 256 outputs) a compute unit, which walks its tiles; the load stream is two
// stages of 64 k ahead of the products and runs on across tile ends, so that only the epilogue's own time stands between two
// tiles.  A stage of 64 KB is requested whole, a request or two between two matrix instructions, into the slot of the ring
// that the stage before last has just left.  Fragments are read by hand, one between every two matrix instructions, a slice
// of 16 k ahead; the schedule is pinned.
//
// Bound by the matrix instructions under the power limit: 8192 x 4096 x 4096 240 us, 1.15 PFLOP/s (a library product of 8192 cubed on
// this card 1.25), 16384 x 1024 x 4096 131 us, 1.05; and by what nothing overlaps, a tile's epilogue: with gelu 165, with 66 MB of
// output for 33 GFLOP 1024 x 512 x 32128 43 (0.79), shaped 80.
//
// Tiles stand in bands of eight rows of tiles, and the columns of a band go to the 8 XCDs in turn, as the blocks do: what the 32
// workers of an XCD have open at a time, 8 row and 4 column tiles, comes into its L2 once, and the XCDs write side by side.
constexpr int kBigM = 256, kBigN = 256;
constexpr int kBigX = kBigM * kStageK * 2, kBigRing = (kBigM + kBigN) * kStageK * 2;       // 32 KB of x rows in a stage of 64 KB
constexpr int kBigStage = 4096;                                                            // a wave's own, for the epilogue
constexpr int kBigLds = 2 * kBigRing + 8 * kBigStage;                                      // all of a compute unit's 160 KB

template <int OFFSET> __device__ __forceinline__ bf16x8 lds_read8(uint32_t at)
{
    bf16x8 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(at), "n"(OFFSET));
    return r;
}

// The epilogue of a wave's 64 x 128: bias and activation where the sums are, then turned through the wave's own 4 KB of LDS, so
// that a lane holds eight consecutive columns of a row.  With no residual bf16 outputs are turned as such, 32 x 64
// at a time, and written in whole lines; fp32 outputs, and those that have a residual before they are rounded,
// 32 x 32 at a time.  16-byte piece c of the 128 bytes of LDS row r lies at c ^ (r & 7).  The LDS accesses are written by hand, so
// that the compiler does not tie them to the requests in flight.
template <class OutT, int FORM>
__device__ __forceinline__ int big_epilogue(const LinearArgs &a, f32x16 (&acc)[2][4], uint32_t stage, int64_t m, int32_t n, int lane)
{
    asm volatile("" : "+v"(lane));           // (its addresses are worked out here: kept over the products they would not fit)
    const int b = lane & 31, h = lane >> 5;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f32x4 add[4];                        // (the bias lies in the wave's LDS)
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\tds_read_b128 %3, %4 offset:96\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(add[0]), "=&v"(add[1]), "=&v"(add[2]), "=&v"(add[3])
                     : "v"(stage + j * 128 + h * 16)
                     : "memory");
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = fmaf(acc[i][j][4 * q + e], a.scale, add[q][e]);
    }
    if (a.act != AS_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 t = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    activate<OutT, 4>(t, a.act, a.act_arg, a.act_inv);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = t[e];
                    __builtin_amdgcn_sched_barrier(0);                // (not more at a time than there are registers for)
                }
    }
    const bool inside = m + 64 <= a.rows && n + 128 <= a.n;
    if constexpr (FORM == 0 && sizeof(OutT) == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int ps = 0; ps < 2; ++ps) {
#pragma unroll
                for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &t = acc[i][ps * 2 + jj];
                        const uint64_t w = (uint64_t)pack2_bf16(t[4 * q + 2], t[4 * q + 3]) << 32 | pack2_bf16(t[4 * q], t[4 * q + 1]);
                        asm volatile("ds_write_b64 %0, %1" ::"v"(stage + b * 128 + (((jj * 4 + q) ^ (b & 7)) << 4) + h * 8), "v"(w)
                                     : "memory");
                    }
                // a lane's pieces are of rows 8 apart, in one column of pieces
                const int row = lane >> 3;
                const uint32_t at = stage + row * 128 + (((lane & 7) ^ row) << 4);
                u32x4_any val[4];
                asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:1024\n\tds_read_b128 %2, %4 offset:2048\n\t"
                             "ds_read_b128 %3, %4 offset:3072\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(val[0]), "=&v"(val[1]), "=&v"(val[2]), "=&v"(val[3])
                             : "v"(at)
                             : "memory");
                const int64_t r = m + i * 32 + row;
                const int32_t col = n + ps * 64 + (lane & 7) * 8;
                OutT *to = (OutT *)a.out + r * a.ldo + col;
#pragma unroll
                for (int p = 0; p < 4; ++p, to += 8 * a.ldo) {
                    if (inside) {
                        *reinterpret_cast<u32x4_any *>(to) = val[p];
                    } else if (r + p * 8 < a.rows) {
                        if (col + 8 <= a.n) {
                            *reinterpret_cast<u32x4_any *>(to) = val[p];
                        } else {
#pragma unroll
                            for (int e = 0; e < 7; ++e) {
                                const uint32_t w = val[p][e >> 1];
                                if (col + e < a.n) to[e] = (OutT)(w >> ((e & 1) * 16));
                            }
                        }
                    }
                }
            }
        return inside ? 16 : -1;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 w = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    asm volatile("ds_write_b128 %0, %1" ::"v"(stage + b * 128 + (((q * 2 + h) ^ (b & 7)) << 4)), "v"(w) : "memory");
                }
                const int row = lane >> 2, c = (lane & 3) * 2;        // (and the row 16 on, of the same swizzle)
                f32x4 t[4];
                asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\t"
                             "s_waitcnt lgkmcnt(0)"
                             : "=&v"(t[0]), "=&v"(t[1]), "=&v"(t[2]), "=&v"(t[3])
                             : "v"(stage + row * 128 + ((c ^ (row & 7)) << 4)), "v"(stage + row * 128 + (((c + 1) ^ (row & 7)) << 4))
                             : "memory");
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    float z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = t[2 * p + (e >> 2)][e & 3];
                    const int64_t r = m + i * 32 + p * 16 + row;
                    const int32_t col = n + j * 32 + c * 4;
                    if (FORM == 0 && inside) store8((OutT *)a.out + r * a.ldo + col, z);
                    else if (r < a.rows && col < a.n) finish8<OutT, FORM == 1, false>(a, r, col, z);
                }
            }
        return FORM == 0 && inside ? 32 : -1;
    }
}

// The epilogue of a wave's 64 x 128 with a shaping.  The sums stay where they are: lane b + 32 h of a 32 x 32 holds row b, columns 8 q + 4 h .. + 3,
// q = 0..3, and everything up to the rounding is done there.  Then lanes exchange halves (v_permlane32_swap, v_permlane16_swap),
// after which a store instruction writes 16 rows of 64 bytes: lane l has row 16 t + l % 16 of store t, and 16 bytes 16 u + 8 h (bf16)
// columns on, u = l / 16 % 2.  No LDS, no waiting.
constexpr uint32_t kOfRows = 512, kOfBits = kOfRows + 5 * 256;       // in the wave's LDS, behind the bias
constexpr uint32_t kOfList = kOfBits + 4 * 256;                       // behind those what seen columns lose, as many as there is room for
constexpr int kListedBig = (kBigStage - (int)kOfList) / 4;

__device__ __forceinline__ uint32_t lds_word(uint32_t at)
{
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(at) : "memory");
    return v;
}
__device__ __forceinline__ float lds_float(uint32_t at) { return __builtin_bit_cast(float, lds_word(at)); }
__device__ __forceinline__ void swap32(uint32_t &x, uint32_t &y)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = r[0];
    y = r[1];
}
__device__ __forceinline__ void swap16(uint32_t &x, uint32_t &y)
{
    const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = r[0];
    y = r[1];
}
// 32 x 32 outputs between the lanes that have the sums and those that meet memory; word w of store t.
struct Turned {
    uint32_t v[2][4];
};
__device__ __forceinline__ void turn(Turned &t)                       // bf16: v[q % 2][...] from [q][word]
{
    // t.v[s][0..1] are quad 2 s, t.v[s][2..3] quad 2 s + 1
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int w = 0; w < 2; ++w) swap32(t.v[s][w], t.v[s][2 + w]);
#pragma unroll
    for (int w = 0; w < 4; ++w) swap16(t.v[0][w], t.v[1][w]);
}
// Requests of what the rows say of a tile's rows m .. m + 63 and columns n .. n + 127, into the wave's LDS, a word of each row a lane.
__device__ __forceinline__ void request_rows(const LinearArgs &a, unsigned char *stage, int64_t m, int32_t n, int lane)
{
    const as_shaping &s = a.shape;
    const int64_t row = m + lane < a.rows ? m + lane : a.rows - 1;
    auto word = [&](const void *p, uint32_t at) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((glb_void *)p, (lds_void *)(stage + at), 4, 0, 0);
    };
    if (s.repetition) word(s.repetition + row, kOfRows);
    if (s.presence) word(s.presence + row, kOfRows + 256);
    if (s.frequency) word(s.frequency + row, kOfRows + 512);
    if (s.bias_ids) word(s.bias_ids + row, kOfRows + 768);
    if (s.mask_ids) word(s.mask_ids + row, kOfRows + 1024);
    if (s.seen) {
        const int32_t words = (a.n + 31) >> 5;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t w = (n >> 5) + e < words ? (n >> 5) + e : words - 1;
            word(s.seen + row * s.seen_ld + w, kOfBits + e * 256);
        }
    }
}

// What a lane has of that, of row b of 32.
struct ShapeTile {
    float repetition, inverse, presence, frequency;
    const float *bias;                        // the row's in the table, from column n on, or null
    bool done;                                // the row is not to be written
    uint32_t seen[4];                         // the bits of its own columns
};
__device__ __forceinline__ int64_t table_row(int64_t id, int64_t rows) { return id < rows ? id : rows - 1; }

// The words of the row's mask.
__device__ __forceinline__ void mask_words(const LinearArgs &a, uint32_t stage, int64_t m, int32_t n, int i, int lane, uint32_t (&mask)[4])
{
    const as_shaping &s = a.shape;
    const int b = lane & 31;
    const int32_t words = (a.n + 31) >> 5;
#pragma unroll
    for (int e = 0; e < 4; ++e) mask[e] = 0xffffffffu;
    if (!s.mask) return;
    const int64_t row = m + i * 32 + b, last = a.rows - 1, mine = row < last ? row : last;
    const int64_t id = table_row(s.mask_ids ? (int32_t)lds_word(stage + kOfRows + 1024 + (uint32_t)(i * 32 + b) * 4) : s.mask_rows == 1 ? 0 : mine, s.mask_rows);
    if (id < 0) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) mask[e] = s.mask[id * s.mask_ld + ((n >> 5) + e < words ? (n >> 5) + e : words - 1)];
}

__device__ __forceinline__ void take_rows(const LinearArgs &a, ShapeTile &t, uint32_t stage, int64_t m, int32_t n, int i, int lane)
{
    const as_shaping &s = a.shape;
    const int b = lane & 31, h = lane >> 5;
    const int64_t row = m + i * 32 + b, last = a.rows - 1, mine = row < last ? row : last;
    const uint32_t at = stage + (uint32_t)(i * 32 + b) * 4;
    t.repetition = s.repetition ? lds_float(at + kOfRows) : 1.f;
    t.presence = s.presence ? lds_float(at + kOfRows + 256) : 0.f;
    t.frequency = s.frequency ? lds_float(at + kOfRows + 512) : 0.f;
    t.inverse = 1.f / t.repetition;
    t.bias = nullptr;
    if (s.bias) {
        const int64_t id = table_row(s.bias_ids ? (int32_t)lds_word(at + kOfRows + 768) : s.bias_rows == 1 ? 0 : mine, s.bias_rows);
        if (id >= 0) t.bias = s.bias + id * s.bias_ld + n;
    }
    t.done = row > last || (s.finished && s.finished[mine]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t left = a.n - n - e * 32;
        t.seen[e] = s.seen && !t.done ? lds_word(at + kOfBits + e * 256) & (0x0f0f0f0fu << 4 * h) : 0u;
        if (left < 32) t.seen[e] &= left > 0 ? (1u << left) - 1u : 0u;
    }
}

// The seen columns of 32 rows from m on, few as a rule and anywhere, listed in the wave's LDS, their counts fetched by the list, all at
// once, and what each is to lose left in its place; a lane's own, `at` on, in the order in which it comes to them.  False where the
// list is too short for them (the first columns of a vocabulary ordered by frequency): then a lane reads the counts of all its columns.
__device__ __forceinline__ bool list_losses(const LinearArgs &a, const ShapeTile &t, uint32_t list, int64_t m, int32_t n, int lane, int &at)
{
    const as_shaping &s = a.shape;
    const int mine = __popc(t.seen[0]) + __popc(t.seen[1]) + __popc(t.seen[2]) + __popc(t.seen[3]);
    const int upto = (int)wave_scan_add((float)mine);
    const int total = __builtin_amdgcn_readlane(upto, 63);
    at = upto - mine;
    if (total > kListedBig) return false;
    uint32_t put = list + (uint32_t)at * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        for (uint32_t w = t.seen[e]; w; w &= w - 1, put += 4)
            asm volatile("ds_write_b32 %0, %1" ::"v"(put), "v"((lane & 31) * 128 + e * 32 + __ffs((int)w) - 1) : "memory");
    for (int k0 = 0; k0 < total; k0 += 2 * kWave) {                   // (the same for the whole wave)
        int32_t place[2], count[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = k0 + k * kWave + lane;
            place[k] = i < total ? (int32_t)lds_word(list + (uint32_t)i * 4) : 0;
            count[k] = 0;
            if (i < total) count[k] = s.counts[(m + (place[k] >> 7)) * s.counts_ld + n + (place[k] & 127)];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = k0 + k * kWave + lane;
            ShapeRow of;
            of.frequency = __shfl(t.frequency, place[k] >> 7, kWave);
            of.presence = __shfl(t.presence, place[k] >> 7, kWave);
            const float less = lost(of, count[k]);
            if (i < total) asm volatile("ds_write_b32 %0, %1" ::"v"(list + (uint32_t)i * 4), "v"(less) : "memory");
        }
    }
    return true;
}

// Gives the number of stores that it has requested last, where that is the same for all lanes, or -1.
// The 32 x 32s go through one piece of code in turn, which is fetched once: unrolled, the epilogue is some 10000 instructions that
// a compute unit comes by twice in a launch, and the first time waits for each line of them.
template <class OutT>
__device__ __forceinline__ int shaped_epilogue(const LinearArgs &a, f32x16 (&acc)[2][4], uint32_t stage, int64_t m, int32_t n, int lane)
{
    asm volatile("" : "+v"(lane));           // (its addresses are worked out here: kept over the products they would not fit)
    const as_shaping &s = a.shape;
    const int b = lane & 31, h = lane >> 5;
    uint32_t masks[2][4];
    mask_words(a, stage, m, n, 0, lane, masks[0]);
    mask_words(a, stage, m, n, 1, lane, masks[1]);
    // a lane's place in the stores: row 16 t + lane % 16, columns from `first` on
    const int u = lane >> 4 & 1, first = sizeof(OutT) == 2 ? 16 * u + 8 * h : 8 * u + 4 * h;
    constexpr int kEach = 16 / (int)sizeof(OutT);                     // columns of a lane's 16 bytes
    bool whole = m + 64 <= a.rows && n + 128 <= a.n;
#pragma unroll 1
    for (int i = 0; i < 2; ++i, m += 32) {
        ShapeTile tile;
        uint64_t skip = 0;
        int at = 0;
        bool listed = true;
        f32x4 more[4];
        auto biases = [&](int j) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t c = j * 32 + 8 * q + 4 * h;
                more[q] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (tile.bias == nullptr) continue;
                if (n + c + 4 <= a.n) {
                    more[q] = *reinterpret_cast<const f32x4_any *>(tile.bias + c);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + c + e < a.n) more[q][e] = tile.bias[c + e];
                }
            }
        };
        i32x4_any all[4];
        auto counts = [&](int j) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t c = n + j * 32 + 8 * q + 4 * h;
                const int32_t *const from = s.counts + (m + b) * s.counts_ld + c;
                all[q] = i32x4_any{0, 0, 0, 0};
                if (tile.done) continue;
                if (c + 4 <= a.n) {
                    all[q] = *reinterpret_cast<const i32x4_any *>(from);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < a.n) all[q][e] = from[e];
                }
            }
        };
        take_rows(a, tile, stage, m - i * 32, n, i, lane);
        skip = __ballot(tile.done);
        whole = whole && skip == 0;
        if (s.bias) biases(0);
        if (s.counts) listed = list_losses(a, tile, stage + kOfList, m, n, lane, at);
        if (!listed) counts(0);
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
            f32x16 &t = acc[0][0];
            f32x4 add[4];                    // (the bias lies in the wave's LDS)
            asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\tds_read_b128 %3, %4 offset:96\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(add[0]), "=&v"(add[1]), "=&v"(add[2]), "=&v"(add[3])
                         : "v"(stage + j * 128 + h * 16)
                         : "memory");
#pragma unroll
            for (int e = 0; e < 16; ++e) t[e] = fmaf(t[e], a.scale, add[e >> 2][e & 3]);
            activate<OutT, 16>(t, a.act, a.act_arg, a.act_inv);
            if (s.seen) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t bits = tile.seen[0] >> (8 * q + 4 * h) & 15u;
                    if (!__any(bits != 0)) continue;
                    f32x4 less = {0.f, 0.f, 0.f, 0.f};
                    if (s.counts && listed) {
                        uint32_t p[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int k = at + __popc(bits & ((1u << e) - 1u));
                            p[e] = stage + kOfList + (uint32_t)(k < kListedBig ? k : kListedBig - 1) * 4;
                        }
                        float l[4];
                        asm volatile("ds_read_b32 %0, %4\n\tds_read_b32 %1, %5\n\tds_read_b32 %2, %6\n\tds_read_b32 %3, %7\n\t"
                                     "s_waitcnt lgkmcnt(0)"
                                     : "=&v"(l[0]), "=&v"(l[1]), "=&v"(l[2]), "=&v"(l[3])
                                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3])
                                     : "memory");
                        less = f32x4{l[0], l[1], l[2], l[3]};
                        at += __popc(bits);
                    } else if (s.counts) {
                        ShapeRow of;
                        of.frequency = tile.frequency;
                        of.presence = tile.presence;
#pragma unroll
                        for (int e = 0; e < 4; ++e) less[e] = lost(of, all[q][e]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = t[4 * q + e], v = fmaf(y, y > 0.f ? tile.inverse : tile.repetition, -less[e]);
                        t[4 * q + e] = bits >> e & 1u ? v : y;
                    }
                }
            }
            if (!listed && j < 3) counts(j + 1);
            if (s.bias) {
#pragma unroll
                for (int e = 0; e < 16; ++e) t[e] += more[e >> 2][e & 3];
                if (j < 3) biases(j + 1);
            }
            if (s.mask) {
                const uint32_t free = masks[0][0] >> 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) t[e] = free >> (8 * (e >> 2) + (e & 3)) & 1u ? t[e] : -__builtin_inff();
            }
#pragma unroll
            for (int half = 0; half < (sizeof(OutT) == 2 ? 1 : 2); ++half) {      // fp32: 32 x 16 at a time
                const int32_t col = n + j * 32 + half * 16 + first, left = a.n - col;
                Turned w;
                if constexpr (sizeof(OutT) == 2) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) w.v[k >> 2][k & 3] = pack2_bf16(t[2 * k], t[2 * k + 1]);
                    turn(w);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float y = t[8 * half + e];
                        w.v[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, y);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) swap16(w.v[0][k], w.v[1][k]);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int in = p * 16 + (lane & 15);
                    const int64_t row = m + in;
                    OutT *const to = (OutT *)a.out + row * a.ldo + col;
                    const u32x4_any v = {w.v[p][0], w.v[p][1], w.v[p][2], w.v[p][3]};
                    if (whole) {
                        *reinterpret_cast<u32x4_any *>(to) = v;
                    } else if (row < a.rows && !(skip >> in & 1u)) {
                        if (left >= kEach) {
                            *reinterpret_cast<u32x4_any *>(to) = v;
                        } else {
#pragma unroll
                            for (int e = 0; e < kEach - 1; ++e)
                                if (e < left) {
                                    const uint32_t x = v[sizeof(OutT) == 2 ? e >> 1 : e];
                                    if constexpr (sizeof(OutT) == 2) to[e] = (OutT)(x >> (e & 1) * 16);
                                    else to[e] = __builtin_bit_cast(OutT, x);
                                }
                        }
                    }
                }
            }
            // the next 32 x 32 takes this one's place
#pragma unroll
            for (int k = 0; k < 3; ++k) acc[0][k] = acc[0][k + 1];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                tile.seen[k] = tile.seen[k + 1];
                masks[0][k] = masks[0][k + 1];
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            acc[0][k] = acc[1][k];
            masks[0][k] = masks[1][k];
        }
    }
    // (loads that were waited for meanwhile only leave less behind)
    return whole ? 8 * (int)sizeof(OutT) : -1;
}

// FORM: what follows the activation, 0 nothing, 1 a residual, 2 a shaping.
template <class OutT, int FORM>
__global__ __launch_bounds__(512, 1) void linear_big(LinearArgs a, uint32_t mtiles, uint32_t ntiles)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kBigLds];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const uint32_t x = blockIdx.x & 7, q = blockIdx.x >> 3, W = gridDim.x >> 3;
    const uint32_t high = mtiles < 8 ? mtiles : 8, low = mtiles % high, bands = mtiles / high;      // the last band has `low` rows of tiles
    const uint32_t columns = bands * ntiles, here = columns > x ? (columns - x + 7) / 8 : 0;        // of whole height; on this XCD
    const uint32_t x2 = (x - columns) & 7, here2 = low && ntiles > x2 ? (ntiles - x2 + 7) / 8 : 0;  // of the last band
    const uint32_t all = here * high + here2 * low;
    if (q >= all) return;
    const uint32_t tiles = (all - q + W - 1) / W;
    auto place = [&](uint32_t j, int64_t &m0, int32_t &n0) __attribute__((always_inline)) {
        uint32_t t = q + j * W;
        if (t < here * high) {
            const uint32_t c = x + 8 * (t / high), band = c / ntiles;
            m0 = (int64_t)(band * high + t % high) * kBigM;
            n0 = (int32_t)((c - band * ntiles) * kBigN);
        } else {
            t -= here * high;
            m0 = (int64_t)(bands * high + t % low) * kBigM;
            n0 = (int32_t)((x2 + 8 * (t / low)) * kBigN);
        }
    };

    // requests: chunk it * 8 + wave of a stage, it 0..3 rows it * 64 + rowb of x, it 4..7 of W; addresses are a uniform base and
    // a lane's 32-bit offset, which changes with the tile only where it has less than 256 rows
    const int rowb = wave * 8 + (lane >> 3);
    const uint32_t piece = (uint32_t)(((lane & 7) ^ ((rowb >> 1) & 7)) << 4);
    const unsigned char *xbase = nullptr, *wbase = nullptr;           // of the tile that is being requested
    uint32_t xoff[4], woff[4];
    auto aim = [&](int64_t m0, int32_t n0) __attribute__((always_inline)) {
        xbase = (const unsigned char *)a.x + m0 * a.ldx * 2;
        wbase = (const unsigned char *)a.W + (int64_t)n0 * a.ldw * 2;
        const int mleft = a.rows - m0 < kBigM ? (int)(a.rows - m0) : kBigM, nleft = a.n - n0 < kBigN ? a.n - n0 : kBigN;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 64 + rowb;
            xoff[it] = (uint32_t)(r < mleft ? r : mleft - 1) * (uint32_t)(a.ldx * 2) + piece;
            woff[it] = (uint32_t)(r < nleft ? r : nleft - 1) * (uint32_t)(a.ldw * 2) + piece;
        }
    };
    const int nstages = a.k / kStageK;                                // at least two
    uint32_t jload = 0;                                               // the tile, and its stage, that is requested next
    int sload = 0;
    auto request1 = [&](int slot, auto it_c) __attribute__((always_inline)) {
        constexpr int it = decltype(it_c)::value;
        unsigned char *const dst = smem + slot * kBigRing + (it * 8 + wave) * 1024;
        if constexpr (it < 4)
            __builtin_amdgcn_global_load_lds((glb_void *)(xbase + (int64_t)sload * (kStageK * 2) + xoff[it]), (lds_void *)dst, 16, 0, 0);
        else
            __builtin_amdgcn_global_load_lds((glb_void *)(wbase + (int64_t)sload * (kStageK * 2) + woff[it - 4]), (lds_void *)dst, 16, 0, 0);
    };
    auto requested = [&]() __attribute__((always_inline)) {           // a whole stage has been: on to the next
        if (++sload == nstages) {
            sload = 0;
            if (++jload < tiles) {
                int64_t m0;
                int32_t n0;
                place(jload, m0, n0);
                aim(m0, n0);
            }
        }
    };

    f32x16 acc[2][4];
    const int frow = lane & 31, fc = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    // (32 rows on are 4 KB on: the swizzle is the same)
    const uint32_t fx = lds0 + (wm * 64 + frow) * 128 + ((fc ^ ((frow >> 1) & 7)) << 4);
    const uint32_t fw = lds0 + kBigX + (wn * 128 + frow) * 128 + ((fc ^ ((frow >> 1) & 7)) << 4);
#define AS_SB() __builtin_amdgcn_sched_barrier(0)
#define AS_RQ(slot_, n_)                                                                                    \
    do {                                                                                                    \
        request1(slot_, std::integral_constant<int, n_>{});                                                 \
        AS_SB();                                                                                            \
    } while (0)
#define AS_RX(f_, i_, so_, kk_)                                                                             \
    do {                                                                                                    \
        f_[i_] = lds_read8<(i_) * 4096>((fx + (so_)) ^ ((kk_) << 5));                                               \
        AS_SB();                                                                                            \
    } while (0)
#define AS_RW(f_, j_, so_, kk_)                                                                             \
    do {                                                                                                    \
        f_[j_] = lds_read8<(j_) * 4096>((fw + (so_)) ^ ((kk_) << 5));                                               \
        AS_SB();                                                                                            \
    } while (0)
#define AS_MM(x_, w_, i_, j_)                                                                               \
    do {                                                                                                    \
        acc[i_][j_] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w_[j_], x_[i_], acc[i_][j_], 0, 0, 0);        \
        AS_SB();                                                                                            \
    } while (0)
    // the fragments are outputs of hand-written reads: the wait is tied to them, so that no product moves above it
#define AS_WAIT(x_, w_)                                                                                     \
    do {                                                                                                    \
        asm volatile("s_waitcnt lgkmcnt(0)"                                                                 \
                     : "+v"(x_[0]), "+v"(x_[1]), "+v"(w_[0]), "+v"(w_[1]), "+v"(w_[2]), "+v"(w_[3]));       \
        AS_SB();                                                                                            \
    } while (0)
    // multiply the slice in (x_, w_) while slice kk_ is read into (nx_, nw_)
#define AS_SLICE(x_, w_, nx_, nw_, so_, kk_)                                                                \
    do {                                                                                                    \
        AS_RX(nx_, 0, so_, kk_); AS_MM(x_, w_, 0, 0); AS_RW(nw_, 0, so_, kk_); AS_MM(x_, w_, 0, 1);         \
        AS_RW(nw_, 1, so_, kk_); AS_MM(x_, w_, 0, 2); AS_RX(nx_, 1, so_, kk_); AS_MM(x_, w_, 0, 3);         \
        AS_RW(nw_, 2, so_, kk_); AS_MM(x_, w_, 1, 0); AS_RW(nw_, 3, so_, kk_); AS_MM(x_, w_, 1, 1);         \
        AS_MM(x_, w_, 1, 2); AS_MM(x_, w_, 1, 3);                                                           \
    } while (0)

    int64_t m0;
    int32_t n0;
    place(0, m0, n0);
    aim(m0, n0);
    AS_RQ(0, 0); AS_RQ(0, 1); AS_RQ(0, 2); AS_RQ(0, 3); AS_RQ(0, 4); AS_RQ(0, 5); AS_RQ(0, 6); AS_RQ(0, 7);
    requested();
    AS_RQ(1, 0); AS_RQ(1, 1); AS_RQ(1, 2); AS_RQ(1, 3); AS_RQ(1, 4); AS_RQ(1, 5); AS_RQ(1, 6); AS_RQ(1, 7);
    requested();
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");                  // stage 0 has landed, stage 1 may still fly
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    bf16x8 xa[2], wa[4], xb[2], wb[4];
    AS_RX(xa, 0, 0u, 0); AS_RX(xa, 1, 0u, 0);
    AS_RW(wa, 0, 0u, 0); AS_RW(wa, 1, 0u, 0); AS_RW(wa, 2, 0u, 0); AS_RW(wa, 3, 0u, 0);
    AS_WAIT(xa, wa);
    int gs = 0;                                                       // stages worked on: stage gs lies in slot gs & 1
    int stores = 0;                                                   // of the tile before, behind the requests for this one
    for (uint32_t j = 0; j < tiles; ++j) {
        place(j, m0, n0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][jj][v] = 0.f;
        for (int s = 0; s < nstages; ++s, ++gs) {
            const int cur = gs & 1;
            const uint32_t so = (uint32_t)cur * kBigRing, son = (uint32_t)(cur ^ 1) * kBigRing;
            const bool more = jload < tiles;
            AS_WAIT(xa, wa);
            AS_SLICE(xa, wa, xb, wb, so, 1);
            AS_WAIT(xb, wb);
            AS_SLICE(xb, wb, xa, wa, so, 2);
            AS_WAIT(xa, wa);
            AS_SLICE(xa, wa, xb, wb, so, 3);
            AS_WAIT(xb, wb);
            // every wave has read all of this stage, and the next one has landed; the stores of the tile before, which were
            // requested after it, may drain on (not in the shaped form, which keeps four registers in memory over the products:
            // the compiler waits for them here, and for the stores with them)
            if (s == 0 && stores == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
            else if (s == 0 && stores == 32) asm volatile("s_waitcnt vmcnt(32)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            AS_SB();
            // the bias of the wave's columns, to where the epilogue finds it: landed before the second stage ends
            if (s == 0) {
                const float *const bias = a.bias + n0 + wn * 128 + lane;
                __builtin_amdgcn_global_load_lds((glb_void *)bias, (lds_void *)(smem + 2 * kBigRing + wave * kBigStage), 4, 0, 0);
                __builtin_amdgcn_global_load_lds((glb_void *)(bias + 64), (lds_void *)(smem + 2 * kBigRing + wave * kBigStage + 256), 4, 0, 0);
                if constexpr (FORM == 2) request_rows(a, smem + 2 * kBigRing + wave * kBigStage, m0 + wm * 64, n0 + wn * 128, lane);
                AS_SB();
            }
            // the last slice, with the first fragments of the next stage (read for nothing behind the last of all) and the requests
            // of the one after it
            AS_RX(xa, 0, son, 0); AS_MM(xb, wb, 0, 0);
            AS_RW(wa, 0, son, 0); AS_MM(xb, wb, 0, 1);
            if (more) AS_RQ(cur, 0);
            AS_RW(wa, 1, son, 0); AS_MM(xb, wb, 0, 2);
            if (more) AS_RQ(cur, 1);
            AS_RX(xa, 1, son, 0); AS_MM(xb, wb, 0, 3);
            if (more) AS_RQ(cur, 2);
            AS_RW(wa, 2, son, 0); AS_MM(xb, wb, 1, 0);
            if (more) AS_RQ(cur, 3);
            AS_RW(wa, 3, son, 0); AS_MM(xb, wb, 1, 1);
            if (more) { AS_RQ(cur, 4); AS_RQ(cur, 5); }
            AS_MM(xb, wb, 1, 2);
            if (more) { AS_RQ(cur, 6); AS_RQ(cur, 7); }
            AS_MM(xb, wb, 1, 3);
            if (more) requested();
        }
        AS_WAIT(xa, wa);                                              // (in flight they must not meet other code)
        const uint32_t stage = lds0 + 2 * kBigRing + (uint32_t)wave * kBigStage;
        if constexpr (FORM == 2) stores = shaped_epilogue<OutT>(a, acc, stage, m0 + wm * 64, n0 + wn * 128, lane);
        else stores = big_epilogue<OutT, FORM>(a, acc, stage, m0 + wm * 64, n0 + wn * 128, lane);
        // the first fragments of the next tile, again (behind the last tile for nothing): they do not take the epilogue's registers.
        // Waited for here: no read is in flight across the loop's end, where the compiler may move registers, or when the wave ends.
        const uint32_t so = (uint32_t)(gs & 1) * kBigRing;
        AS_RX(xa, 0, so, 0); AS_RX(xa, 1, so, 0);
        AS_RW(wa, 0, so, 0); AS_RW(wa, 1, so, 0); AS_RW(wa, 2, so, 0); AS_RW(wa, 3, so, 0);
        AS_WAIT(xa, wa);
    }
#undef AS_SB
#undef AS_RQ
#undef AS_RX
#undef AS_RW
#undef AS_MM
#undef AS_WAIT
#undef AS_SLICE
}

// ---------------------------------------------------------------- fp32

// A block, four waves as WM x WN x KG (KG shares of the sum, as above), takes TM x TN outputs, KS k of each share at a time:
// v_mfma_f32_16x16x4_f32, W first (lane l has k = l / 16 of row l % 16 of either operand, and of the result row l % 16, columns
// 4 (l / 16) .. + 3).  Which k are a lane's first to fourth of sixteen does not matter as long as both operands agree, so a
// lane takes four in a row with one read, of LDS rows 16 bytes longer than they need be (no two lanes of 16 on one bank).
// Rows of x and W may start anywhere: 16 bytes at a time through registers, the next step's while this one is worked on.
// Large products run at 70 % of the fp32 matrix rate (2048 x 1024 x 2048 80 us, 107 TFLOP/s), small ones wait for their loads
// (333 x 515 x 1031 10 us, 16 x 512 x 2048 3.9).
template <int WM, int WN, int KG, int FM, int FN, int KS>
__global__ __launch_bounds__(256) void linear_f32(LinearArgs a, uint32_t mtiles, uint32_t ntiles)
{
    static_assert(WM * WN * KG == 4 && KS % 16 == 0, "four waves, whole groups of 16 k");
    constexpr int TM = WM * FM * 16, TN = WN * FN * 16, kRows = TM + TN, kStep = KG * KS;
    constexpr int kRow = kStep + 4;                                   // floats of an LDS row
    constexpr int kMine = kRows * kStep / 4 / 256;                    // pieces of four k that a thread moves
    static_assert(kRows * kStep % 1024 == 0, "the same for all threads");
    typedef TileEnd<float, TM, TN, KG> End;
    constexpr int kLds = 2 * kRows * kRow * 4 > End::kBytes ? 2 * kRows * kRow * 4 : End::kBytes;
    static_assert(kLds <= 160 * 1024, "LDS");
    __shared__ __attribute__((aligned(16))) unsigned char smem[kLds];
    float *const lds = reinterpret_cast<float *>(smem);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
    const uint32_t bid = blockIdx.x, eight = bid / (8 * mtiles), in = bid % (8 * mtiles);
    const uint32_t across = ntiles - eight * 8 < 8 ? ntiles - eight * 8 : 8;
    const int32_t n0 = (int32_t)((eight * 8 + in % across) * TN);
    const int64_t m0 = (int64_t)(in / across) * TM;

    const float *from[kMine];                                         // rows past either end repeat the last
    int k_of[kMine], at[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int u = tid + i * 256, r = u / (kStep / 4);
        k_of[i] = u % (kStep / 4) * 4;
        at[i] = r * kRow + k_of[i];
        if (r < TN) {
            const int32_t n = n0 + r < a.n ? n0 + r : a.n - 1;
            from[i] = (const float *)a.W + (int64_t)n * a.ldw;
        } else {
            const int64_t m = m0 + r - TN < a.rows ? m0 + r - TN : a.rows - 1;
            from[i] = (const float *)a.x + m * a.ldx;
        }
    }
    f32x4 next[kMine];
    auto request = [&](int k0) __attribute__((always_inline)) {
        if (k0 + kStep <= a.k) {                                      // (the same for all)
#pragma unroll
            for (int i = 0; i < kMine; ++i) next[i] = *reinterpret_cast<const f32x4_any *>(from[i] + k0 + k_of[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kMine; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = k0 + k_of[i] + e;
                    const float v = from[i][k < a.k ? k : a.k - 1];
                    next[i][e] = k < a.k ? v : 0.f;
                }
        }
    };
    TileEnd<float, TM, TN, KG> end;
    request(0);
    end.first(a, m0, n0);
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int fw = (wn * FN * 16 + (lane & 15)) * kRow + kg * KS + (lane >> 4) * 4;
    const int fx = (TN + wm * FM * 16 + (lane & 15)) * kRow + kg * KS + (lane >> 4) * 4;
    int slot = 0;
    for (int k0 = 0; k0 < a.k; k0 += kStep, slot ^= 1) {
        float *const here = lds + slot * kRows * kRow;
#pragma unroll
        for (int i = 0; i < kMine; ++i) *reinterpret_cast<f32x4 *>(here + at[i]) = next[i];
        if (k0 + kStep < a.k) request(k0 + kStep);
        __syncthreads();
#pragma unroll
        for (int g = 0; g < KS / 16; ++g) {
            f32x4 w[FN], x[FM];
#pragma unroll
            for (int j = 0; j < FN; ++j) w[j] = *reinterpret_cast<const f32x4 *>(here + fw + j * 16 * kRow + g * 16);
#pragma unroll
            for (int i = 0; i < FM; ++i) x[i] = *reinterpret_cast<const f32x4 *>(here + fx + i * 16 * kRow + g * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j][e], x[i][e], acc[i][j], 0, 0, 0);
        }
    }
    end.second(a);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            *reinterpret_cast<f32x4 *>(lds + (kg * TM + (wm * FM + i) * 16 + (lane & 15)) * End::kStride + (wn * FN + j) * 16 + 4 * (lane >> 4)) =
                acc[i][j];
    __syncthreads();
    end.finish(a, lds);
}

// ---------------------------------------------------------------- layer

// The layer's bias in fp32, zeros behind it up to a whole number of 256 columns (and everywhere, where it has none); and the
// weights in rows of kp, zeros behind k, where the caller's rows are not of that kind.
template <class T> __global__ __launch_bounds__(256) void layer_bias_kernel(const T *bias, float *out, int32_t n, int32_t padded)
{
    const int32_t i = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (i < padded) out[i] = bias && i < n ? widen(bias[i]) : 0.f;
}
// eight elements a thread, `pieces` of them a row
__global__ __launch_bounds__(256) void layout_kernel(const uint16_t *in, int64_t ld, int64_t rows, int32_t k, uint16_t *out, uint32_t pieces)
{
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i >> 32 ? (int64_t)(i / pieces) : (int64_t)((uint32_t)i / pieces);
    const int32_t c = (int32_t)(i - row * pieces) * 8;
    if (row >= rows) return;
    const uint16_t *const from = in + row * ld + c;
    u32x4_any v = {0, 0, 0, 0};
    if (c + 8 <= k) {
        v = fetch16<false>(from);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < k) v[e >> 1] |= (uint32_t)from[e] << (e & 1) * 16;
    }
    put16<false>(out + row * (int64_t)pieces * 8 + c, v);
}

static as_status launch_layout(as_ctx *ctx, hipStream_t stream, const void *in, int64_t ld, int64_t rows, int32_t k, void *out, int32_t kp)
{
    const int64_t blocks = (rows * (kp / 8) + 255) / 256;
    if (blocks > 0x7fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "too large to lay out");
    hipLaunchKernelGGL(layout_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, (const uint16_t *)in, ld, rows, k, (uint16_t *)out,
                       (uint32_t)(kp / 8));
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
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
        const as_status st = launch_layout(nullptr, nullptr, W, ldw, l.n, l.k, l.own, l.kp);
        if (st != AS_OK) return st;
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

template <class OutT, int WAVES, int KW, int U> static as_status launch_few(as_ctx *ctx, const LinearArgs &a)
{
    constexpr int TN = WAVES / KW * 16;
    launch(ctx, kKernelLogits, linear_few<OutT, WAVES, KW, U>, dim3((unsigned)((a.n + TN - 1) / TN)), dim3(WAVES * kWave), 0, a);
    return AS_OK;
}

template <class OutT> static as_status launch_big(as_ctx *ctx, const LinearArgs &a)
{
    const uint32_t mtiles = (uint32_t)((a.rows + kBigM - 1) / kBigM), ntiles = (uint32_t)((a.n + kBigN - 1) / kBigN);
    const dim3 grid((unsigned)(ctx->num_cus / 8 * 8));
    if (a.shaped) launch(ctx, kKernelLogits, linear_big<OutT, 2>, grid, dim3(512), 0, a, mtiles, ntiles);
    else if (a.residual) launch(ctx, kKernelLogits, linear_big<OutT, 1>, grid, dim3(512), 0, a, mtiles, ntiles);
    else launch(ctx, kKernelLogits, linear_big<OutT, 0>, grid, dim3(512), 0, a, mtiles, ntiles);
    return AS_OK;
}

// Whether the kernel for large products can take it: two stages of K, 32-bit offsets inside a tile.
static bool big_applies(const as_ctx *ctx, const LinearArgs &a)
{
    return a.k >= 2 * kStageK && ctx->num_cus >= 8 && !(a.shaped && a.residual) && a.ldx < (1 << 22) && a.ldw < (1 << 22) &&
           (a.rows + kBigM - 1) / kBigM * ((a.n + kBigN - 1) / kBigN) < (1LL << 30);
}

// Which form a product takes: the least of these times, in us, with S stages of 64 k, lines fitted to the launches below on 256
// compute units; where the wide ones differ little their order does not matter.  A tile of 32 x 32 whose four waves share the
// sum has the shortest way through a long one; with two blocks a compute unit (Many) it takes more tiles; 64 x 64 has
// less traffic, alone with more on its way, or five blocks a unit; 128 x 128 and the large one less again.
//            rows k n      32   32 Many  64   64 Many  128   large
//      64  512   2048     3.8    3.7    5.1    4.9    9.4   18.7
//      64 1024   8192     9.4    6.2    7.5   10.5   14.3   27.8
//     128 2048   2048     7.7    8.0   11.0   17.0   24.4   44.7
//     256 1024   4096    17.2   10.7    7.8   10.5   15.9   28.2
//    1024 2048    512    14.5    9.7   11.3   17.5   24.6   45.4
//    1024  512   2048    23.5   14.2    7.6    7.8   11.8   19.8
//    2048  512   2048    44.4   25.4   13.3   12.0   13.1   20.6
//    2048 2048   2048    99.8   78.2   36.3   32.4   29.1   47.1
//     128  512  32128    44.7   25.8   13.8   12.6   13.9   22.2
//    1024  512  32128     390    235   94.4   83.2   93.5   50
//    4096 1024   4096     249    168   84.0   68.6   73.4   41.0
// A shaping adds to what a block does behind its sums: 64 x 512 x 32128 21.8 / 13.5 / 13.4 / 19.6 / 42.8 (32 Many, 64, 64 Many, 128,
// large), 256 x 512 x 32128 - / 39.1 / 29.4 / 53.2 / 45.4, 1024 x 512 x 32128 - / 153 / 117 / 211 / 80.
// Up to 16 rows (us, by 2, 4 and 8 shares of the sum, then 32 Many and 64 Many): 1 x 512 x 2048 3.1 / 3.1 / 4.5 / 3.6 / 4.5, 1 x
// 512 x 8192 3.8 / 4.7 / 7.3 / 4.6 / 6.3, 1 x 4096 x 4096 16.2 / 9.5 / 8.1 / 13.8 / 29.9, 16 x 2048 x 512 9.0 / 5.8 / 5.9 / 6.3 / 9.9, 1 x
// 1024 x 256000 85.2 / 78.8 / 152 / 97.3 / 88.9, 16 x 512 x 32128 9.6 / 16.7 / 31.5 / 9.3 / 7.6, 16 x 1024 x 256000 127 / 126 / 230 / 111 / 95.4:
// many rows over many columns read x once too often.
enum Form { kByRule, kTile32, kTile32Many, kTile64, kTile64Many, kTile128, kBig, kFew2, kFew4, kFew8, kForms };

static Form form_of(const as_ctx *ctx, const LinearArgs &a)
{
    if (ctx->linear_shape > kByRule && ctx->linear_shape < kForms) {
        const Form f = (Form)ctx->linear_shape;
        const bool can = f == kBig ? big_applies(ctx, a) : f < kFew2 || a.rows <= 16;
        if (can) return f;
    }
    const double S = (double)a.k / kStageK, cus = ctx->num_cus > 0 ? ctx->num_cus : 1;
    if (a.rows <= 4 || (a.rows <= 16 && a.n <= 8192)) return S >= 48 ? kFew8 : S >= 16 || a.n <= 4096 ? kFew4 : kFew2;
    auto units = [&](int64_t t) { return ceil((double)((a.rows + t - 1) / t) * (double)((a.n + t - 1) / t) / cus); };      // tiles a compute unit
    const double u32 = units(32), u64 = units(64), u128 = units(128), u256 = units(256), more = a.shaped ? 1.0 : 0.0;
    const double few = u64 < 5 ? u64 : 5, full = (double)((a.rows + 255) / 256) * (double)((a.n + 255) / 256) / cus;
    const double t[] = {
        1.2 + u32 * (1.2 + 0.16 * S) + more * (4.0 + 0.6 * u32),
        1.2 + (u32 <= 1 ? 0.7 : ceil(u32 / 2)) * (0.9 + 0.26 * S) + more * (4.0 + 0.6 * u32),
        2.6 + 0.26 * S + (u64 - 1) * (0.9 + 0.235 * S) + more * (4.5 + 1.85 * u64),
        2.2 + 0.46 * S + (few - 1) * (0.6 + 0.14 * S) + (u64 - few) * (0.75 + 0.225 * S) + more * (4.0 + u64),
        1.0 + u128 * (7.2 + 0.6 * S + 15.0 * more),
        5.0 + u256 * (4.0 + 1.1 * S + 0.7 * S * (full < 1 ? full : 1) + 17.0 * more),
    };
    int best = 0;
    for (int f = 1; f < 6; ++f)
        if (t[f] < t[best] && (f < 5 || big_applies(ctx, a))) best = f;
    return (Form)(best + 1);
}

template <class OutT> static as_status launch_bf16(as_ctx *ctx, const LinearArgs &a)
{
    switch (form_of(ctx, a)) {
    case kTile32: return launch_tile<OutT, 1, 1, 4, 1, 1, 4>(ctx, a);
    case kTile32Many: return launch_tile<OutT, 1, 1, 4, 1, 1, 2>(ctx, a);
    case kTile64: return launch_tile<OutT, 2, 2, 1, 1, 1, 4>(ctx, a);
    case kTile128: return launch_tile<OutT, 2, 2, 1, 2, 2, 4>(ctx, a);
    case kBig: return launch_big<OutT>(ctx, a);
    case kFew2: return launch_few<OutT, 4, 2, 4>(ctx, a);
    case kFew4: return launch_few<OutT, 4, 4, 4>(ctx, a);
    case kFew8: return launch_few<OutT, 8, 8, 4>(ctx, a);
    default: return launch_tile<OutT, 2, 2, 1, 1, 1, 2>(ctx, a);
    }
}

template <int WM, int WN, int KG, int FM, int FN, int KS> static as_status launch_f32_tile(as_ctx *ctx, const LinearArgs &a)
{
    constexpr int TM = WM * FM * 16, TN = WN * FN * 16;
    const int64_t mtiles = (a.rows + TM - 1) / TM, ntiles = (a.n + TN - 1) / TN;
    if (mtiles * ntiles > 0x7fffffffLL || mtiles > 0x0fffffffLL) return fail(ctx, AS_ERR_UNSUPPORTED, "product too large for one launch");
    launch(ctx, kKernelLogits, linear_f32<WM, WN, KG, FM, FN, KS>, dim3((unsigned)(mtiles * ntiles)), dim3(256), 0, a, (uint32_t)mtiles,
           (uint32_t)ntiles);
    return AS_OK;
}

// The same for fp32, by lines fitted to these (us, S stages of 64 k, tiles of 16 x 16 / 16 x 32 / 32 x 64 / 64 x 64 / 128 x 128): 1 x 515 x
// 1031 4.5 / 5.4 / 9.7 / 14.4 / 40.0; 16 x 512 x 2048 3.8 / 4.6 / 8.8 / 13.3 / 38.6; 16 x 55 x 32128 9.3 / 6.5 / 5.8 / 7.1 / 9.7; 128 x 2048 x
// 512 8.9 / 13.6 / 28.5 / 46.0 / 146; 333 x 515 x 1031 12.3 / 9.8 / 10.6 / 16.2 / 49.5; 512 x 512 x 2048 - / 18.1 / 15.2 / 15.2 / 42.3; 1024 x
// 512 x 2048 - / 31.6 / 25.9 / 25.0 / 42.8; 2048 x 1024 x 2048 - / 111 / 89.9 / 82.3 / 80.3; 4000 x 40 x 6000 - / 117 / 59.7 / 56.4 / 50.6.
static as_status launch_fp32(as_ctx *ctx, const LinearArgs &a)
{
    const double S = (double)a.k / kStageK, cus = ctx->num_cus > 0 ? ctx->num_cus : 1;
    auto units = [&](int64_t tm, int64_t tn) { return ceil((double)((a.rows + tm - 1) / tm) * (double)((a.n + tn - 1) / tn) / cus); };
    const double t[] = {
        2.4 + 0.19 * S + (units(16, 16) - 1) * (0.9 + 0.09 * S),
        2.6 + 0.36 * S + (units(16, 32) - 1) * (0.3 + 0.19 * S),
        3.2 + 0.78 * S + (units(32, 64) - 1) * (0.3 + 0.66 * S),
        3.2 + 1.35 * S + (units(64, 64) - 1) * (0.3 + 1.2 * S),
        4.0 + units(128, 128) * (5.0 + 4.5 * S),
    };
    int best = 0;
    for (int f = 1; f < 5; ++f)
        if (t[f] < t[best]) best = f;
    if (ctx->linear_shape > 0 && ctx->linear_shape <= 5) best = ctx->linear_shape - 1;
    switch (best) {
    case 0: return launch_f32_tile<1, 1, 4, 1, 1, 32>(ctx, a);
    case 1: return launch_f32_tile<1, 1, 4, 1, 2, 16>(ctx, a);
    case 2: return launch_f32_tile<1, 2, 2, 2, 2, 16>(ctx, a);
    case 3: return launch_f32_tile<2, 2, 1, 2, 2, 32>(ctx, a);
    default: return launch_f32_tile<2, 2, 1, 4, 4, 16>(ctx, a);
    }
}

as_status launch_linear(as_ctx *ctx, const as_layer *l, LinearArgs a)
{
    as_status st = AS_OK;
    if (l->wdtype == AS_F32) {
        st = launch_fp32(ctx, a);
    } else {
        if (!x_as_it_is(l, a.x, a.ldx)) {
            st = launch_layout(ctx, ctx->stream, a.x, a.ldx, a.rows, l->k, ctx->linear_x.ptr, l->kp);
            if (st != AS_OK) return st;
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
