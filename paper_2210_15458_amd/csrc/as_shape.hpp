// Modifiers of logits, eight consecutive ones of a row at a time: what as_shape_logits applies to logits that are there and
// the layers' epilogue to those it has just summed.
#pragma once

#include "as_common.hpp"

namespace as {

// 16 bytes at any address that its elements may have: the card reads and writes them in one instruction all the same
// (a few cycles more where they lie across two lines), so rows that start anywhere need no form of their own.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi)
{
    uint32_t r;
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(lo), "v"(hi));
    return r;
}

// Eight logits from and to memory; `left` of them (at least one) lie in the row.
__device__ __forceinline__ void load8(const uint16_t *p, int left, float (&y)[8])
{
    if (left >= 8) {
        const u32x4_any v = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = v[e];
            y[2 * e] = __builtin_bit_cast(float, w << 16);
            y[2 * e + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = e < left ? __builtin_bit_cast(float, (uint32_t)p[e] << 16) : 0.f;
    }
}
__device__ __forceinline__ void load8(const float *p, int left, float (&y)[8])
{
    if (left >= 8) {
        const f32x4_any a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = a[e];
            y[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = e < left ? p[e] : 0.f;
    }
}
__device__ __forceinline__ void store8(uint16_t *p, int left, const float (&y)[8])
{
    u32x4_any v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack2_bf16(y[2 * e], y[2 * e + 1]);
    if (left >= 8) {
        *reinterpret_cast<u32x4_any *>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = v[e >> 1];
            if (e < left) p[e] = (uint16_t)(w >> ((e & 1) * 16));
        }
    }
}
__device__ __forceinline__ void store8(float *p, int left, const float (&y)[8])
{
    if (left >= 8) {
        f32x4_any a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] = y[e];
            b[e] = y[4 + e];
        }
        *reinterpret_cast<f32x4_any *>(p) = a;
        *reinterpret_cast<f32x4_any *>(p + 4) = b;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = y[e];
    }
}

// What one row of a shaping comes to.
struct ShapeRow {
    const uint32_t *seen, *mask;       // null: none
    const int32_t *counts;
    const float *bias;
    float repetition, presence, frequency;
};

__device__ __forceinline__ ShapeRow shape_row(const as_shaping &s, int64_t row)
{
    ShapeRow r;
    r.seen = s.seen ? s.seen + row * s.seen_ld : nullptr;
    r.counts = s.counts ? s.counts + row * s.counts_ld : nullptr;
    r.repetition = s.repetition ? s.repetition[row] : 1.f;
    r.presence = s.presence ? s.presence[row] : 0.f;
    r.frequency = s.frequency ? s.frequency[row] : 0.f;
    r.bias = nullptr;
    r.mask = nullptr;
    if (s.bias) {
        int64_t id = s.bias_ids ? s.bias_ids[row] : s.bias_rows == 1 ? 0 : row;
        id = id < s.bias_rows ? id : s.bias_rows - 1;
        if (id >= 0) r.bias = s.bias + id * s.bias_ld;
    }
    if (s.mask) {
        int64_t id = s.mask_ids ? s.mask_ids[row] : s.mask_rows == 1 ? 0 : row;
        id = id < s.mask_rows ? id : s.mask_rows - 1;
        if (id >= 0) r.mask = s.mask + id * s.mask_ld;
    }
    return r;
}

// Columns col .. col + 7 of the row (col a multiple of 8, so their bits lie in one byte of a word), `left` of them inside it.
__device__ __forceinline__ void shape8(const ShapeRow &r, int32_t col, int left, float (&y)[8])
{
    if (r.seen) {
        uint32_t b = (r.seen[col >> 5] >> (col & 24)) & 0xffu;
        if (left < 8) b &= (1u << left) - 1u;
        if (b) {
            int32_t n[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] = 0;
            if (r.counts) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (b >> e & 1u) n[e] = r.counts[col + e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (b >> e & 1u) {
                    float v = y[e];
                    v = v > 0.f ? v / r.repetition : v * r.repetition;
                    v -= r.frequency * (float)n[e];
                    y[e] = n[e] > 0 ? v - r.presence : v;
                }
        }
    }
    if (r.bias) {
        float add[8];
        load8(r.bias + col, left, add);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += add[e];
    }
    if (r.mask) {
        const uint32_t b = r.mask[col >> 5] >> (col & 24);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = b >> e & 1u ? y[e] : -__builtin_inff();
    }
}

}  // namespace as
