// Logits shaped by penalties, biases and masks, and the record of tokens that the penalties go by.
#include "as_shape.hpp"

namespace as {

// ---------------------------------------------------------------- logits

// A block takes 2048 columns of a row, a thread eight at a time.
template <class T>
__global__ __launch_bounds__(256) void shape_kernel(as_shaping s, const T *in, int64_t rows, int64_t ld, T *out, int64_t ldo,
                                                    int32_t V, int32_t chunks)
{
    const int64_t items = rows * chunks;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int64_t row = i / chunks;
        const int32_t col = (int32_t)(i - row * chunks) * 2048 + (int32_t)threadIdx.x * 8;
        if (s.finished && s.finished[row]) continue;
        if (col >= V) continue;
        const ShapeRow r = shape_row(s, row);
        float y[8];
        load8(in + row * ld + col, V - col, y);
        shape8(r, col, V - col, y);
        store8(out + row * ldo + col, V - col, y);
    }
}

as_status launch_shape(as_ctx *ctx, const as_shaping &s, const void *logits, int64_t rows, int64_t ld, void *out, int64_t ldo)
{
    const int32_t chunks = (ctx->V + 2047) / 2048;
    const int64_t items = rows * chunks;
    const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20));
    if (ctx->dtype == AS_BF16)
        hipLaunchKernelGGL(shape_kernel<uint16_t>, grid, dim3(256), 0, ctx->stream, s, (const uint16_t *)logits, rows, ld,
                           (uint16_t *)out, ldo, ctx->V, chunks);
    else
        hipLaunchKernelGGL(shape_kernel<float>, grid, dim3(256), 0, ctx->stream, s, (const float *)logits, rows, ld,
                           (float *)out, ldo, ctx->V, chunks);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

// ---------------------------------------------------------------- history

// A block sets kSlice tokens of a row's record: it counts in LDS those of the row's lists that fall into its slice (whole
// numbers: the order of the additions does not matter), then writes the slice's bits, and the counts of those tokens that
// are or were seen; all others are zero and stay so.  So the counts, 4 bytes a token of the vocabulary, are touched only
// where something is, and a launch needs nothing cleared before it.
constexpr int kSlice = 8192, kSetThreads = 512;
constexpr uint32_t kOfPrompt = 0x80000000u;      // beside the count: the prompt has the token

__global__ __launch_bounds__(kSetThreads) void history_set_kernel(HistoryArgs a, int32_t slices)
{
    __shared__ uint32_t count[kSlice];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t items = a.rows * slices;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int64_t row = i / slices;
        const int32_t first = (int32_t)(i - row * slices) * kSlice;
        if (a.which && !a.which[row]) continue;                       // (the same for the whole block)
        const int32_t width = a.V - first < kSlice ? a.V - first : kSlice;
        for (int v = tid; v < kSlice; v += kSetThreads) count[v] = 0;
        __syncthreads();
        if (a.prompts) {
            const int64_t p = row / a.per;
            int64_t from = a.offsets[p], to = a.offsets[p + 1];
            from = from > 0 ? from : 0;
            to = to < a.prompts_len ? to : a.prompts_len;
            for (int64_t j = from + tid; j < to; j += kSetThreads) {
                const uint32_t u = (uint32_t)a.prompts[j] - (uint32_t)first;
                if (u < (uint32_t)width) atomicOr(&count[u], kOfPrompt);
            }
        }
        if (a.tokens) {
            int32_t n = a.lens ? a.lens[row] : a.T;
            n = n < a.T ? n : a.T;
            const int32_t *mine = a.tokens + row * a.tokens_ld;
            for (int32_t j = tid; j < n; j += kSetThreads) {
                const uint32_t u = (uint32_t)mine[j] - (uint32_t)first;
                if (u < (uint32_t)width) atomicAdd(&count[u], 1u);
            }
        }
        __syncthreads();
        uint32_t *const words = a.seen + row * a.seen_ld + first / 32;
        int32_t *const counts = a.counts ? a.counts + row * a.counts_ld + first : nullptr;
        for (int v0 = wave * kWave; v0 < width; v0 += kSetThreads) {
            const int v = v0 + lane;
            const uint32_t c = count[v];
            const uint64_t now = __ballot(c != 0);
            if (v < width) {
                const bool was = words[v >> 5] >> (v & 31) & 1u;
                if (counts && (was || (c & ~kOfPrompt))) counts[v] = (int32_t)(c & ~kOfPrompt);
            }
            if ((lane & 31) == 0 && v < width) words[v >> 5] = (uint32_t)(now >> lane);
        }
        __syncthreads();
    }
}

as_status launch_history_set(as_ctx *ctx, const HistoryArgs &a)
{
    const int32_t slices = (a.V + kSlice - 1) / kSlice;
    const int64_t items = a.rows * slices;
    hipLaunchKernelGGL(history_set_kernel, dim3((unsigned)(items < (1 << 20) ? items : 1 << 20)), dim3(kSetThreads), 0, ctx->stream, a,
                       slices);
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
