// Modifiers of logits, eight consecutive ones of a row at a time: what as_shape_logits applies to logits that are there and
// the layers' epilogue to those it has just summed.
#pragma once

#include <type_traits>

#include "as_common.hpp"

namespace as {

// 16 bytes at any address that its elements may have: the card reads and writes them in one instruction all the same
// (a few cycles more where they lie across two lines), so rows that start anywhere need no form of their own.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi)
{
    uint32_t r;
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(lo), "v"(hi));
    return r;
}

// Eight logits from and to memory.  NT: past the caches.
template <class T> struct Raw8;
template <> struct Raw8<uint16_t> {
    u32x4_any v;
};
template <> struct Raw8<float> {
    f32x4_any v[2];
};
template <bool NT, class E> __device__ __forceinline__ auto fetch16(const E *p)
{
    typedef std::conditional_t<sizeof(E) == 2, u32x4_any, f32x4_any> V;
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else return *reinterpret_cast<const V *>(p);
}
template <bool NT, class E, class V> __device__ __forceinline__ void put16(E *p, V v)
{
    typedef std::conditional_t<sizeof(E) == 2, u32x4_any, f32x4_any> A;
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<A *>(p));
    else *reinterpret_cast<A *>(p) = v;
}
template <bool NT = false> __device__ __forceinline__ void load_raw8(const uint16_t *p, Raw8<uint16_t> &r) { r.v = fetch16<NT>(p); }
template <bool NT = false> __device__ __forceinline__ void load_raw8(const float *p, Raw8<float> &r)
{
    r.v[0] = fetch16<NT>(p);
    r.v[1] = fetch16<NT>(p + 4);
}
__device__ __forceinline__ void widen8(const Raw8<uint16_t> &r, float (&y)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t w = r.v[e];
        y[2 * e] = __builtin_bit_cast(float, w << 16);
        y[2 * e + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<float> &r, float (&y)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = r.v[e >> 2][e & 3];
}
template <bool NT = false> __device__ __forceinline__ void store8(uint16_t *p, const float (&y)[8])
{
    u32x4_any v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack2_bf16(y[2 * e], y[2 * e + 1]);
    put16<NT>(p, v);
}
template <bool NT = false> __device__ __forceinline__ void store8(float *p, const float (&y)[8])
{
    f32x4_any a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = y[e];
        b[e] = y[4 + e];
    }
    put16<NT>(p, a);
    put16<NT>(p + 4, b);
}
// single ones
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t h) { return __builtin_bit_cast(float, (uint32_t)h << 16); }
__device__ __forceinline__ void store1(uint16_t *p, float y) { *p = (uint16_t)pack2_bf16(y, y); }
__device__ __forceinline__ void store1(float *p, float y) { *p = y; }

// Read-only memory that a whole block reads at one place: by scalar loads, which go beside the vector memory's queue.
template <class T> __device__ __forceinline__ T scalar_load(const T *p)
{
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)p;
}
template <bool UNIFORM, class T> __device__ __forceinline__ T row_load(const T *p)
{
    if constexpr (UNIFORM) return scalar_load(p);
    else return *p;
}

// What one row of a shaping comes to.
struct ShapeRow {
    const uint32_t *seen, *mask;       // null: none
    const int32_t *counts;
    const float *bias;
    float repetition, inverse, presence, frequency;      // inverse: 1 / repetition, which a positive logit is multiplied by
};

// UNIFORM: the row is the same for all lanes.
template <bool UNIFORM> __device__ __forceinline__ ShapeRow shape_row(const as_shaping &s, int64_t row)
{
    ShapeRow r;
    r.seen = s.seen ? s.seen + row * s.seen_ld : nullptr;
    r.counts = s.counts ? s.counts + row * s.counts_ld : nullptr;
    r.repetition = s.repetition ? row_load<UNIFORM>(s.repetition + row) : 1.f;
    r.inverse = 1.f / r.repetition;
    r.presence = s.presence ? row_load<UNIFORM>(s.presence + row) : 0.f;
    r.frequency = s.frequency ? row_load<UNIFORM>(s.frequency + row) : 0.f;
    r.bias = nullptr;
    r.mask = nullptr;
    if (s.bias) {
        int64_t id = s.bias_ids ? row_load<UNIFORM>(s.bias_ids + row) : s.bias_rows == 1 ? 0 : row;
        id = id < s.bias_rows ? id : s.bias_rows - 1;
        if (id >= 0) r.bias = s.bias + id * s.bias_ld;
    }
    if (s.mask) {
        int64_t id = s.mask_ids ? row_load<UNIFORM>(s.mask_ids + row) : s.mask_rows == 1 ? 0 : row;
        id = id < s.mask_rows ? id : s.mask_rows - 1;
        if (id >= 0) r.mask = s.mask + id * s.mask_ld;
    }
    return r;
}

// What a seen logit loses by its count.
__device__ __forceinline__ float lost(const ShapeRow &r, int32_t count)
{
    return count > 0 ? fmaf(r.frequency, (float)count, r.presence) : r.frequency * (float)count;
}

// One logit: seen, its count, its bias, whether it is free.
__device__ __forceinline__ float shape1(const ShapeRow &r, bool seen, int32_t count, float bias, bool free, float y)
{
    y = seen ? fmaf(y, y > 0.f ? r.inverse : r.repetition, -lost(r, count)) : y;
    y += bias;
    return free ? y : -__builtin_inff();
}

// Eight columns of a row, col .. col + 7 (col a multiple of 8, so their bits lie in one byte of a word; all inside the row), in
// three stages, so that a thread with several can have the loads of all of them on their way before it waits for one: what
// the row says of them, the counts of those that are seen, and the logits themselves.
struct Shape8 {
    uint32_t seen, mask;
    f32x4_any bias[2];
    int32_t count[8];
};

__device__ __forceinline__ void shape8_request(const ShapeRow &r, int32_t col, Shape8 &p)
{
    if (r.seen) p.seen = r.seen[col >> 5];
    if (r.mask) p.mask = r.mask[col >> 5];
    if (r.bias) {
        p.bias[0] = *reinterpret_cast<const f32x4_any *>(r.bias + col);
        p.bias[1] = *reinterpret_cast<const f32x4_any *>(r.bias + col + 4);
    }
}
__device__ __forceinline__ void shape8_counts(const ShapeRow &r, int32_t col, Shape8 &p)
{
    if (!r.seen) return;
    p.seen = p.seen >> (col & 24) & 0xffu;
#pragma unroll
    for (int e = 0; e < 8; ++e) p.count[e] = 0;
    if (r.counts) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (p.seen >> e & 1u) p.count[e] = r.counts[col + e];
    }
}
__device__ __forceinline__ void shape8_apply(const ShapeRow &r, int32_t col, const Shape8 &p, float (&y)[8])
{
    if (r.seen) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = shape1(r, p.seen >> e & 1u, p.count[e], 0.f, true, y[e]);
    }
    if (r.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += p.bias[e >> 2][e & 3];
    }
    if (r.mask) {
        const uint32_t b = p.mask >> (col & 24);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = b >> e & 1u ? y[e] : -__builtin_inff();
    }
}

// One column of a row, for the last few of a row.
__device__ __forceinline__ float shape_one(const ShapeRow &r, int32_t col, float y)
{
    const bool seen = r.seen && (r.seen[col >> 5] >> (col & 31) & 1u);
    const int32_t count = seen && r.counts ? r.counts[col] : 0;
    return shape1(r, seen, count, r.bias ? r.bias[col] : 0.f, !r.mask || (r.mask[col >> 5] >> (col & 31) & 1u), y);
}

}  // namespace as
