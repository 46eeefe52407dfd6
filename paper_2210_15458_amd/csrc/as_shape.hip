// Logits shaped by penalties, biases and masks, and the record of tokens that the penalties go by.
#include "as_shape.hpp"

namespace as {

// ---------------------------------------------------------------- logits

// A wave takes P * 512 columns of one row, a lane P times eight of them, each a load of 16 bytes (bf16) 1 KB apart, and has
// nothing to do with the others of its block.  Columns past the row's last whole eight are read there again and not written, so
// that all loads of a lane stand in one piece of code; the V % 8 columns behind it are single ones, a lane each, of the
// row's last wave.
//
// The bits of the wave's columns (seen, free) are read once, a word a lane, and handed round.  Few tokens of a row are seen,
// anywhere in it; a lane that looked up the counts of its own eight would wait for them one after another, for the sake
// of one or two lanes of its wave.  So the seen columns are listed in LDS first, their counts fetched by the list, all at
// once, and what each is to lose (frequency * count, and presence) left in its place, where the column's lane finds it
// by the number of seen columns before it.  Where more are seen than the list holds, the lanes read all their counts.
// Bound by the memory: 1024 x 32128 bf16 in and out 28 us without penalties (4.7 TB/s), 1024 x 256000 170 (6.2); the counts add a line of
// 128 bytes for each seen token that no other shares one with: with 16, 64, 256, 2000 tokens counted and as many of a prompt 32,
// 34, 44, 51 us, and with all modifiers 48 (256 of either) and 263 (512).
constexpr int kListed = 256;
template <class T, int P, bool NT>
__global__ __launch_bounds__(256) void shape_kernel(as_shaping s, const T *in, int64_t rows, int64_t ld, T *out, int64_t ldo,
                                                    int32_t V)
{
    constexpr int kCols = P * 512, kWords = kCols / 32;
    static_assert(kWords <= kWave, "a word a lane");
    __shared__ int32_t lists[4][kListed + 8];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t *const list = lists[wave];
    const int32_t base = ((int32_t)blockIdx.x * 4 + wave) * kCols, whole = V & ~7, words = (V + 31) >> 5;
    if (base >= V) return;
    const int32_t mine = (base >> 5) + lane, left = V - mine * 32;
    const bool has = lane < kWords && mine < words;
    // bits past V are nobody's
    const uint32_t valid = !has || left >= 32 ? 0xffffffffu : (1u << left) - 1u;
    int32_t col[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        col[p] = base + p * 512 + lane * 8;
        col[p] = col[p] < whole ? col[p] : whole - 8;
    }
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        if (s.finished && s.finished[row]) continue;
        const T *const from = in + row * ld;
        T *const to = out + row * ldo;
        Raw8<T> raw[P];
        if (whole > 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) load_raw8<NT>(from + col[p], raw[p]);
        }
        const ShapeRow r = shape_row<true>(s, row);
        uint32_t seen = 0, mask = 0;
        if (r.seen && has) seen = r.seen[mine] & valid;
        if (r.mask && has) mask = r.mask[mine];
        f32x4_any bias[P][2];
        if (r.bias && whole > 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                bias[p][0] = *reinterpret_cast<const f32x4_any *>(r.bias + col[p]);
                bias[p][1] = *reinterpret_cast<const f32x4_any *>(r.bias + col[p] + 4);
            }
        }
        int before = 0, total = 0;                 // seen columns before this lane's word, in all of them
        if (r.counts) {
            const int n = __popc(seen);
            const int upto = (int)wave_scan_add((float)n);            // (at most 2048: exact in the scan's floats)
            before = upto - n;
            total = __builtin_amdgcn_readlane(upto, 63);
            if (total <= kListed) {
                int at = before;
                for (uint32_t w = seen; w; w &= w - 1) list[at++] = lane * 32 + __ffs((int)w) - 1;
                __builtin_amdgcn_wave_barrier();
                for (int i = lane; i < total; i += kWave)
                    list[i] = __builtin_bit_cast(int32_t, lost(r, r.counts[base + list[i]]));
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (whole > 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int word = p * 16 + (lane >> 2), byte = (lane & 3) * 8;
                float y[8];
                widen8(raw[p], y);
                if (r.seen) {
                    const uint32_t w = (uint32_t)__shfl((int)seen, word, kWave), b = w >> byte;
                    float less[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) less[e] = 0.f;
                    if (r.counts && total <= kListed) {
                        int at = __shfl(before, word, kWave) + __popc(w & ((1u << byte) - 1u));
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            less[e] = __builtin_bit_cast(float, list[at]);
                            at += b >> e & 1u;
                        }
                    } else if (r.counts) {
                        const i32x4_any c0 = *reinterpret_cast<const i32x4_any *>(r.counts + col[p]),
                                        c1 = *reinterpret_cast<const i32x4_any *>(r.counts + col[p] + 4);
#pragma unroll
                        for (int e = 0; e < 8; ++e) less[e] = lost(r, e < 4 ? c0[e & 3] : c1[e & 3]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float v = fmaf(y[e], y[e] > 0.f ? r.inverse : r.repetition, -less[e]);
                        y[e] = b >> e & 1u ? v : y[e];
                    }
                }
                if (r.bias) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += bias[p][e >> 2][e & 3];
                }
                if (r.mask) {
                    const uint32_t b = (uint32_t)__shfl((int)mask, word, kWave) >> byte;
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = b >> e & 1u ? y[e] : -__builtin_inff();
                }
                if (base + p * 512 + lane * 8 < whole) store8<NT>(to + col[p], y);
            }
        }
        const int32_t c = whole + lane;
        if (c < V && base <= whole && whole < base + kCols) store1(to + c, shape_one(r, c, widen(from[c])));
        __builtin_amdgcn_wave_barrier();
    }
}

template <class T, int P, bool NT>
static void shape_rows(as_ctx *ctx, const as_shaping &s, const void *logits, int64_t rows, int64_t ld, void *out, int64_t ldo)
{
    const dim3 grid((unsigned)((ctx->V + P * 2048 - 1) / (P * 2048)), (unsigned)smaller(rows, 65535));
    hipLaunchKernelGGL((shape_kernel<T, P, NT>), grid, dim3(256), 0, ctx->stream, s, (const T *)logits, rows, ld, (T *)out, ldo, ctx->V);
}

template <class T>
static void shape_rows(as_ctx *ctx, const as_shaping &s, const void *logits, int64_t rows, int64_t ld, void *out, int64_t ldo)
{
    const bool nt = stream_rows(rows, ld, sizeof(T));
    if (rows * ((ctx->V + 4095) / 4096) < 2 * (int64_t)ctx->num_cus) shape_rows<T, 1, false>(ctx, s, logits, rows, ld, out, ldo);
    else if (nt) shape_rows<T, 2, true>(ctx, s, logits, rows, ld, out, ldo);
    else shape_rows<T, 2, false>(ctx, s, logits, rows, ld, out, ldo);
}

as_status launch_shape(as_ctx *ctx, const as_shaping &s, const void *logits, int64_t rows, int64_t ld, void *out, int64_t ldo)
{
    if (ctx->dtype == AS_BF16) shape_rows<uint16_t>(ctx, s, logits, rows, ld, out, ldo);
    else shape_rows<float>(ctx, s, logits, rows, ld, out, ldo);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

// ---------------------------------------------------------------- history

// A block sets kSlice tokens of a row's record: it marks and counts in LDS those of the row's lists that fall into its slice
// (whole numbers: the order of the additions does not matter), then writes the slice's words of bits, a lane each, and the
// counts of those tokens that are or were seen; all others are zero and stay so.  So the counts, 4 bytes a token of the
// vocabulary, are touched only where something is, and a launch needs nothing cleared before it.  Every block
// reads its rows' whole lists: they are short beside the record, and come from the caches.  16 prompts of up to 512 tokens, 64 rows
// each with up to 64 of its own, V = 32128: 18 us, four rows a block; 16 rows of a prompt of up
// to 32768 with up to 4096 of their own, V = 256000: 12 us, which every block reads.  Slices of 4096: 24 and 18 us, of 16384 the
// same as these; a row's old words and tokens asked for a row ahead: the same.
constexpr int kSlice = 8192;

// A token's count in LDS: the 32 of a word turned by the word's number, so that lanes at one bit of their words meet no bank twice
__device__ __forceinline__ uint32_t count_at(uint32_t u) { return (u & ~31u) | ((u + (u >> 5)) & 31u); }

// Marks n tokens in the slice, and counts them if COUNT; four tokens a lane and load, four loads on their way.
template <bool COUNT>
__device__ __forceinline__ void tally(const int32_t *tokens, int64_t n, int32_t first, int32_t width, uint32_t *bits, uint32_t *count)
{
    auto one = [&](int32_t t) __attribute__((always_inline)) {
        const uint32_t u = (uint32_t)t - (uint32_t)first;
        if (u < (uint32_t)width) {
            atomicOr(&bits[u >> 5], 1u << (u & 31));
            if constexpr (COUNT) atomicAdd(&count[count_at(u)], 1u);
        }
    };
    if (n < 4) {
        if (threadIdx.x < n) one(tokens[threadIdx.x]);
        return;
    }
    const int64_t step = (int64_t)blockDim.x * 4;
    auto some = [&](int64_t j, auto quads) __attribute__((always_inline)) {
        constexpr int Q = decltype(quads)::value;
        i32x4_any t[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int64_t at = j + q * step < n - 4 ? j + q * step : n - 4;      // (the last four again: those not yet taken count)
            t[q] = *reinterpret_cast<const i32x4_any *>(tokens + at);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int64_t from = j + q * step, at = from < n - 4 ? from : n - 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e >= from) one(t[q][e]);
        }
    };
    if (n <= step) some((int64_t)threadIdx.x * 4, std::integral_constant<int, 1>{});
    else
        for (int64_t j = (int64_t)threadIdx.x * 4; j < n; j += 4 * step) some(j, std::integral_constant<int, 4>{});
}

// A block's rows, `group` of them, are of one prompt, whose tokens it marks once.
template <int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void history_set_kernel(HistoryArgs a, int32_t group, int32_t groups)
{
    constexpr int kWords = kSlice / 32;
    static_assert(WAVES * kWave % kWords == 0 && 32 % (WAVES * kWave / kWords) == 0, "a word a thread, or a part");
    __shared__ __attribute__((aligned(16))) uint32_t count[kSlice];
    __shared__ uint32_t bits[kWords];
    const int tid = threadIdx.x;
    const int32_t first = (int32_t)blockIdx.x * kSlice, width = a.V - first < kSlice ? a.V - first : kSlice;
    // at the end a word of bits is a thread's, or with more threads than words a part of it
    constexpr int kParts = WAVES * kWave / kWords;
    const int word = tid / kParts;
    const uint32_t part = (uint32_t)((1ull << (32 / kParts)) - 1) << (tid % kParts * (32 / kParts));
    const int64_t items = (a.rows + a.per - 1) / a.per * groups;
    for (int64_t item = blockIdx.y; item < items; item += gridDim.y) {
        const int64_t p = item / groups, row0 = p * a.per + (item - p * groups) * group;
        int64_t row1 = row0 + group < (p + 1) * a.per ? row0 + group : (p + 1) * a.per;
        row1 = row1 < a.rows ? row1 : a.rows;
        if (row0 >= row1) continue;                                   // (the last prompt may have fewer rows)
        if (tid < kWords) bits[tid] = 0;
        for (int v = tid * 4; v < kSlice; v += WAVES * kWave * 4) *reinterpret_cast<uint4 *>(count + v) = uint4{0, 0, 0, 0};
        __syncthreads();
        uint32_t of_prompt = 0;
        if (a.prompts) {
            int64_t from = scalar_load(a.offsets + p), to = scalar_load(a.offsets + p + 1);
            from = from > 0 ? from : 0;
            to = to < a.prompts_len ? to : a.prompts_len;
            if (from < to) tally<false>(a.prompts + from, to - from, first, width, bits, count);
            __syncthreads();
            if (tid < kWords) of_prompt = bits[tid];
            __syncthreads();                                          // (before the first row's own tokens are marked in the same words)
        }
        for (int64_t row = row0; row < row1; ++row) {
            if (a.which && !a.which[row]) continue;                   // (the same for the whole block)
            uint32_t *const words = a.seen + row * a.seen_ld + first / 32;
            const uint32_t was = word * 32 < width ? words[word] : 0u;
            if (a.tokens) {
                int32_t n = a.lens ? scalar_load(a.lens + row) : a.T;
                n = n < a.T ? n : a.T;
                const int32_t *const mine = a.tokens + row * a.tokens_ld;
                if (n > 0 && a.counts) tally<true>(mine, n, first, width, bits, count);
                else if (n > 0) tally<false>(mine, n, first, width, bits, count);
                __syncthreads();
            }
            if (word * 32 < width) {
                const uint32_t now = bits[word];
                if (a.counts) {
                    int32_t *const counts = a.counts + row * a.counts_ld + first + word * 32;
                    for (uint32_t w = (now | was) & part; w; w &= w - 1) {
                        const int b = __ffs((int)w) - 1;
                        if (word * 32 + b >= width) continue;
                        uint32_t *const c = count + count_at((uint32_t)(word * 32 + b));
                        counts[b] = (int32_t)*c;
                        *c = 0;                                       // as the next row finds it
                    }
                }
                if (tid % kParts == 0) words[word] = now;
            }
            __syncthreads();
            if (tid < kWords) bits[tid] = of_prompt;
            __syncthreads();
        }
    }
}

as_status launch_history_set(as_ctx *ctx, const HistoryArgs &a)
{
    const int64_t slices = (a.V + kSlice - 1) / kSlice, prompts = (a.rows + a.per - 1) / a.per;
    // long lists: more threads to read them, and a block a compute unit
    const int64_t length = (a.prompts ? a.prompts_len / prompts : 0) + (a.tokens ? a.T : 0);
    const bool many = length > 4096;
    // rows that share a block, where there are blocks enough
    int64_t group = a.prompts ? slices * a.rows / ((many ? 1 : 4) * (int64_t)ctx->num_cus) : 1;
    group = group < 1 ? 1 : group > a.per ? a.per : group;
    const int64_t groups = (a.per + group - 1) / group;
    const dim3 grid((unsigned)slices, (unsigned)smaller(prompts * groups, 65535));
    if (many) hipLaunchKernelGGL(history_set_kernel<16>, grid, dim3(16 * kWave), 0, ctx->stream, a, (int32_t)group, (int32_t)groups);
    else hipLaunchKernelGGL(history_set_kernel<4>, grid, dim3(4 * kWave), 0, ctx->stream, a, (int32_t)group, (int32_t)groups);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

// One token more a row: a row is one thread's, so nothing is contended.
__global__ __launch_bounds__(256) void history_add_kernel(HistoryArgs a, const int32_t *tokens, const uint8_t *finished)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows || (finished && finished[row])) return;
    const int32_t t = tokens[row];
    if (t < 0 || t >= a.V) return;
    a.seen[row * a.seen_ld + (t >> 5)] |= 1u << (t & 31);
    if (a.counts) ++a.counts[row * a.counts_ld + t];
}

as_status launch_history_add(as_ctx *ctx, const HistoryArgs &a, const int32_t *tokens, const uint8_t *finished)
{
    hipLaunchKernelGGL(history_add_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, ctx->stream, a, tokens, finished);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

}  // namespace as
