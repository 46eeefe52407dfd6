// A paged cache of keys and values, and the attention that reads it.
//
// Row r's query at position i over keys j:  s_j = scale q.k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  m = max_j s_j, over
// the j that it sees (j <= i; with a window j > i - window or j < sinks).  Keys are taken a tile at a time, with the running m,
// l = sum exp(s_j - m) and O = sum exp(s_j - m) v_j; a tile that raises m by d multiplies l and O by exp(-d).  Parts of the keys that
// different waves or blocks have taken are joined the same way:  m = max m_a, l = sum l_a exp(m_a - m), O = sum O_a exp(m_a - m).
#include <type_traits>

#include "as_shape.hpp"

namespace as {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kNone = -__builtin_inff();

// Scores are products until they are weighed: a weight is 2^((q.k - m) scale), m the largest q.k (of a negative scale's negated queries),
// with log2(e) in the scale.  The difference is taken first: of a score times the scale and a rounded maximum times the scale what is
// left is the product's rounding, which passes 2^127 where scores do 2^31.
__device__ __forceinline__ float weight_scale(const AttendArgs &a) { return a.scale == 0.f ? 1.f : fabsf(a.scale); }      // (above 0; 0: the queries are zeros)

// Two weights as bf16.  (By the compiler, not the instruction by hand: what an exponential has just left may be read by other
// instructions only after a pause that the compiler sees to.)
__device__ __forceinline__ uint32_t weights2(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// ---------------------------------------------------------------- which queries, which keys

// Ragged queries go by tiles of `rows` rows (a row: one head of those that share a key head, of one token); sequence s has the
// slots floor(offsets[s] * group / rows) + s on, one a tile: never fewer than its tiles, and in order, so a block finds
// its sequence by a search in the offsets alone.
__device__ __forceinline__ int64_t offset_at(const AttendArgs &a, int64_t s)
{
    const int64_t o = a.offsets[s];
    return o < 0 ? 0 : o > a.tokens ? a.tokens : o;
}
// The last sequence whose first slot is at most `slot` (ROWS 0: whose first token is), and its tokens; 64 of them looked at at once.
struct Found {
    int64_t s, from, to;
};
template <int ROWS> __device__ __forceinline__ Found find_sequence(const AttendArgs &a, int64_t slot, uint32_t group, uint32_t rows = ROWS)
{
    int64_t lo = 0, hi = a.rows;                       // the answer is in [lo, hi)
    for (;;) {
        const int64_t step = hi - lo > 63 ? (hi - lo + 62) / 63 : 1, s = lo + lane_id() * step;
        const uint64_t o = s <= a.rows ? offset_at(a, s) : 0;
        const bool behind = s < hi && (int64_t)(ROWS > 0 ? o * group / rows + s : o) <= slot;
        int n = __popcll(__ballot(behind));            // (monotone: the first n lanes; the first of all in any case)
        n = n > 0 ? n : 1;
        lo += (n - 1) * step;
        if (step == 1) {                               // (n is at most 63)
            const uint32_t low = (uint32_t)o, high = (uint32_t)(o >> 32);
            Found f;
            f.s = lo;
            f.from = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, n - 1) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, n - 1));
            f.to = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, n) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, n));
            return f;
        }
        hi = lo + step < hi ? lo + step : hi;
    }
}

// What a block works on: up to ROWS queries that share a key head, and a segment of keys.
struct Work {
    int32_t head;                 // key head
    const int32_t *table;         // the segment's pages
    int32_t n;                    // its keys
    int32_t key0;                 // position of its first key
    // of a lane's query: whether there is one, its token and head, its position relative to the segment's first key
    bool valid;
    int64_t token;
    int32_t qhead, at;
    // the smallest and largest position of the block's queries, and of those of the lane's wave (none: -1 as the largest)
    int32_t lo, hi, wave_lo, wave_hi;
};

__device__ __forceinline__ int32_t length_of(const int32_t *lens, int64_t i, int32_t room)
{
    const int32_t n = scalar_load(lens + i);
    return n < 0 ? 0 : n > room ? room : n;
}

// Query `mine` of the ROWS of an item, for a wave that has EACH of them from wave_from on.  False where the block has nothing to
// do.  (The launch sees to it that a sequence's queries times the heads of a group fit 32 bits.)
template <int ROWS, int EACH, int MODE>
__device__ __forceinline__ bool find_work(const AttendArgs &a, const AttendPiece &piece, uint32_t mine, uint32_t wave_from, uint32_t item, Work &w)
{
    const uint32_t G = a.group;
    // x / G for x < G + 128
    auto by_group = [&](uint32_t x) __attribute__((always_inline)) { return x * a.group_inverse >> 24; };
    if constexpr (MODE == kAttendRagged) {
        const uint32_t slot = item / (uint32_t)a.kv_heads;
        w.head = (int32_t)(item - slot * a.kv_heads);
        const Found f = find_sequence<ROWS>(a, slot, G);
        const int32_t len = length_of(a.lens, f.s, a.room);
        const int64_t first = ((int64_t)slot - f.s - (int64_t)((uint64_t)f.from * G / ROWS)) * ROWS;      // the tile's first row in its sequence
        const int64_t all = (f.to - f.from) * G;
        // (below 0: offsets that fall)
        if (first < 0 || first >= all || (a.finished && a.finished[f.s])) return false;
        w.table = a.table + f.s * a.table_ld;
        w.n = len;
        w.key0 = 0;
        const uint32_t first_token = (uint32_t)first / G, rest = (uint32_t)first - first_token * G;
        const uint32_t left = all - first < ROWS ? (uint32_t)(all - first) : ROWS;
        w.valid = mine < left;
        const uint32_t x = rest + (w.valid ? mine : left - 1), i = by_group(x);
        int32_t first_at = len - (int32_t)(f.to - f.from) + (int32_t)first_token;
        first_at = first_at > -ROWS ? first_at : -ROWS;        // (below 0 the item's queries see nothing, however far; and a window off it fits 32 bits)
        w.token = f.from + first_token + i;
        w.qhead = (int32_t)(w.head * G + x - i * G);
        w.at = first_at + (int32_t)i;
        const uint32_t wave_to = wave_from + EACH < left ? wave_from + EACH : left;
        w.lo = first_at;
        w.hi = first_at + (int32_t)by_group(rest + left - 1);
        w.wave_lo = first_at + (int32_t)by_group(rest + wave_from);
        w.wave_hi = wave_from < left ? first_at + (int32_t)by_group(rest + wave_to - 1) : -1;
        return true;
    }
    const uint32_t group = MODE == kAttendOwn && piece.tiles == 1 ? item : item / (uint32_t)piece.tiles, tile = item - group * piece.tiles;
    const uint32_t p = group / (uint32_t)a.kv_heads;    // row or prompt
    w.head = (int32_t)(group - p * a.kv_heads);
    if constexpr (MODE == kAttendOwn) {
        if (a.finished && a.finished[p]) return false;
        const uint32_t g = tile * ROWS + mine;
        w.valid = g < G;
        w.token = p;
        w.qhead = (int32_t)(w.head * G + g);
        w.table = a.table + p * a.table_ld;
        w.n = length_of(a.lens, p, a.room);
        w.key0 = a.prompt_table ? length_of(a.prompt_lens, p / (uint32_t)a.per, a.prompt_room) : 0;
        w.at = w.lo = w.hi = w.wave_lo = w.wave_hi = w.n - 1;
        return true;
    }
    w.table = a.prompt_table + p * a.prompt_table_ld;
    w.n = length_of(a.prompt_lens, p, a.prompt_room);
    w.key0 = 0;
    const uint32_t first = tile * ROWS, first_row = first / G, x = first - first_row * G + mine, c = by_group(x);
    const int64_t row = (int64_t)p * a.per + first_row + c;
    w.valid = first_row + c < (uint32_t)a.per && row < a.rows;
    if (w.valid && a.finished && a.finished[row]) w.valid = false;
    w.token = row;
    w.qhead = (int32_t)(w.head * G + x - c * G);
    w.at = w.lo = w.hi = w.wave_lo = w.n - 1;
    w.wave_hi = first + wave_from < (uint32_t)a.per * G ? w.n - 1 : -1;
    if (a.window > 0) {
        // rows are as far behind their prompt as they have tokens of their own (without a window they see all of it)
        int32_t own = 0;
        if (w.valid && a.table) {
            own = a.lens[row];
            own = own < 0 ? 0 : own > a.room ? a.room : own;
        }
        w.at += own;
        int32_t lo = w.valid ? w.at : 0x7fffffff, hi = w.valid ? w.at : -1;
#pragma unroll
        for (int d = 1; d < EACH; d <<= 1) {
            const int32_t u = __shfl_xor(lo, d, kWave), v = __shfl_xor(hi, d, kWave);
            lo = u < lo ? u : lo;
            hi = v > hi ? v : hi;
        }
        w.lo = w.wave_lo = __builtin_amdgcn_readfirstlane(lo);
        w.hi = w.wave_hi = __builtin_amdgcn_readfirstlane(hi);
        if (ROWS > EACH) {
            __shared__ int32_t ends[2][4];
            const int wave = threadIdx.x >> 6;
            if (lane_id() == 0) {
                ends[0][wave] = lo;
                ends[1][wave] = hi;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w.lo = ends[0][i] < w.lo ? ends[0][i] : w.lo;
                w.hi = ends[1][i] > w.hi ? ends[1][i] : w.hi;
            }
            w.lo = __builtin_amdgcn_readfirstlane(w.lo);
            w.hi = __builtin_amdgcn_readfirstlane(w.hi);
        }
        if (w.lo > w.hi) w.lo = w.hi;                  // (no query)
        if (w.wave_lo > w.wave_hi) w.wave_lo = w.wave_hi;
    }
    return true;
}

// The tiles of BN keys that some query of a block may see, and this part's share of them.
struct Keys {
    int32_t n, lo_at, hi_at;      // keys; smallest and largest position of the queries
    int32_t lo, hi;               // the keys seen by some query: [lo, hi) and [0, sinks)
    int32_t window, sinks;
    int32_t sink_tiles, main_tile, first, last;
    __device__ __forceinline__ int32_t base(int32_t t, int32_t BN) const { return (t < sink_tiles ? t : t - sink_tiles + main_tile) * BN; }
    // every query sees every key of the tile
    __device__ __forceinline__ bool whole(int32_t b, int32_t BN) const
    {
        return b + BN <= n && b + BN - 1 <= lo_at && (window <= 0 || b > hi_at - window || b + BN <= sinks);
    }
    __device__ __forceinline__ bool seen(int32_t t, int32_t at) const
    {
        return t < n && t <= at && (window <= 0 || t > at - window || t < sinks);
    }
    __device__ __forceinline__ bool seen_by_some(int32_t t) const { return t < hi && (t >= lo || t < sinks); }
};

__device__ __forceinline__ Keys keys_of(const AttendArgs &a, const Work &w, int32_t lo_at, int32_t hi_at, int32_t BN, int32_t part, int32_t parts,
                                        int32_t least)
{
    Keys k;
    k.n = w.n;
    k.lo_at = lo_at;
    k.hi_at = hi_at;
    k.window = a.window;
    k.sinks = a.sinks - w.key0;
    k.hi = w.n < hi_at + 1 ? w.n : hi_at + 1;
    k.hi = k.hi > 0 ? k.hi : 0;
    k.lo = a.window > 0 && lo_at - a.window + 1 > 0 ? lo_at - a.window + 1 : 0;
    k.lo = k.lo < k.hi ? k.lo : k.hi;
    const int32_t first = k.sinks < 0 ? 0 : k.sinks < k.lo ? k.sinks : k.lo;
    k.sink_tiles = (first + BN - 1) / BN;
    k.main_tile = k.lo / BN;
    if (k.sink_tiles >= k.main_tile) k.sink_tiles = k.main_tile = 0;
    const int32_t count = k.sink_tiles + (k.hi + BN - 1) / BN - k.main_tile;
    int32_t share = (count + parts - 1) / parts;
    share = share > least ? share : least;
    k.first = part * share < count ? part * share : count;
    k.last = count - k.first < share ? count : k.first + share;
    return k;
}

// Address of a key head's token t.
__device__ __forceinline__ const char *token_at(const void *cache, const AttendArgs &a, const Work &w, int32_t t, int32_t esz)
{
    int32_t page = w.table[t >> a.page_shift];
    page = page < 0 ? 0 : page < a.pages ? page : a.pages - 1;
    return (const char *)cache + (uint64_t)(uint32_t)page * a.page_bytes +
           (((int64_t)w.head << a.page_shift) + (t & ((1 << a.page_shift) - 1))) * (int64_t)(a.dim * esz);
}

// The words' values that are no numbers (infinities, NaN): whether there are any, from the largest magnitudes; and the words without.
template <class T> __device__ __forceinline__ uint32_t larger_magnitude(uint32_t a, uint32_t x)
{
    if constexpr (sizeof(T) == 2) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, x & 0x7fff7fffu)));
    } else {
        x &= 0x7fffffffu;
        return a > x ? a : x;
    }
}
template <class T> __device__ __forceinline__ bool no_number(uint32_t a)
{
    return a >= 0x7f800000u || (sizeof(T) == 2 && (a & 0xffffu) >= 0x7f80u);
}
template <class T> __device__ __forceinline__ uint32_t numbers(uint32_t x)
{
    const uint32_t high = (x & 0x7f800000u) == 0x7f800000u ? 0u : sizeof(T) == 2 ? x & 0xffff0000u : x;
    return sizeof(T) == 2 ? high | ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) : high;
}

// What a wave left out of its product: the values that are no numbers in the tiles that not every query sees whole, to the sums of
// those that do see them (0 * NaN is NaN, so the product cannot leave them out by their weight).
template <class T, int QUERIES>
__device__ __forceinline__ void add_odd_values(const AttendArgs &a, const Work &w, const Keys &keys, int32_t BN, int32_t from, int32_t every, int32_t at,
                                               float *sums, int32_t stride, int32_t d0, int32_t d1)
{
    for (int32_t t = keys.first + from; t < keys.last; t += every) {
        const int32_t base = keys.base(t, BN);
        if (keys.whole(base, BN)) continue;
        for (int32_t x = base; x < base + BN && x < keys.hi; ++x) {
            if (!keys.seen_by_some(x)) continue;
            const T *const row = (const T *)token_at(a.v, a, w, x, sizeof(T));
            for (int32_t first = d0; first < d1; first += kWave) {
                const int32_t d = first + lane_id();
                const float y = d < d1 ? widen(row[d]) : 0.f;
                const bool is = (__builtin_bit_cast(uint32_t, y) & 0x7f800000u) == 0x7f800000u;
                if (!__any(is)) continue;
#pragma unroll 1
                for (int q = 0; q < QUERIES; ++q)
                    if (keys.seen(x, __builtin_amdgcn_readlane(at, q)) && is) sums[q * stride + d - d0] += y;
            }
        }
    }
}

// ---------------------------------------------------------------- 16 queries a block, keys straight from memory

// A wave takes tiles of keys from memory to registers, 16 queries at a time (of one key head: the heads of a row that share it, or
// rows of a prompt, or tokens of a sequence), the four waves of a block every fourth tile, joined at the end.  Both products are
// taken transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane's scores, its share of P^T and its sums all are of one query
// (lane % 16), whose m and l it carries.  A lane of quarter q = lane / 16 gets from the first product the scores of tokens
// 16 a + 4 q + j (a: 16 tokens of the tile, j < 4), and hands them to the second as its share of the sum over tokens, which may go
// in any order as long as V^T's lanes have the same tokens: so V is read in whole rows, 16 lanes one token, and the 2-byte
// values of a lane's tokens are put in pairs by byte permutations, without LDS.
// Bound by the memory where rows are long (8 rows of up to 65536 tokens, 8 key heads of 128, bf16: 295 us, 5.3 TB/s, and 7 us of joining;
// 256 rows that see 1028 each 101 us, 5.7), by one tile after the other where they are short (about 1.1 us each).  A tile's keys are asked for as soon as
// the scores of the one before it are taken, its values behind that one's product, into the same registers (305 -> 301, fp32 prompts 35 -> 32).
template <class T, int DP> struct AttendForm;
template <int DP> struct AttendForm<uint16_t, DP> {
    static constexpr int kSub = 2, kKey = DP / 32, kVBytes = DP == 64 ? 8 : 16, kChunks = DP == 256 ? 2 : 1, kEach = kVBytes / 2;
};
template <int DP> struct AttendForm<float, DP> {
    static constexpr int kSub = 1, kKey = DP / 16, kVBytes = DP == 96 ? 8 : 16, kEach = kVBytes / 4, kChunks = DP / (16 * kEach);
};

// Of the dimensions that come to a form of DP the fewest: which of a row's pieces may lie past its end.
template <class T, int DP>
constexpr int kLeastDim = DP == 64 ? 8 : sizeof(T) == 2 ? DP / 2 + 8 : DP == 96 ? 72 : DP == 128 ? 104 : DP == 192 ? 136 : 200;

// Two, four or eight values after each other.
__device__ __forceinline__ void store_some(float *p, const float (&y)[2])
{
    typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
    *reinterpret_cast<f32x2_any *>(p) = f32x2{y[0], y[1]};
}
__device__ __forceinline__ void store_some(float *p, const float (&y)[4]) { *reinterpret_cast<f32x4_any *>(p) = f32x4{y[0], y[1], y[2], y[3]}; }
__device__ __forceinline__ void store_some(uint16_t *p, const float (&y)[4])
{
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<u32x2_any *>(p) = u32x2{weights2(y[0], y[1]), weights2(y[2], y[3])};
}
template <class T> __device__ __forceinline__ void store_some(T *p, const float (&y)[8]) { store8(p, y); }

template <class T, int DP> struct RowsShared {
    static constexpr int kStride = DP + 4;
    __attribute__((aligned(16))) float sums[4 * 16 * kStride];
    float2 stats[4][16];
    int64_t token[16];                                 // of each query, -1: none ...
    int32_t head[16];                                  // ... and its head
};

template <class T, int DP, bool FULL, bool BYPAGE, int WAVES, int MODE>
__device__ __forceinline__ void attend_rows(const AttendArgs &a, const AttendPiece &piece, uint32_t item, int32_t part, RowsShared<T, DP> &shared)
{
    typedef AttendForm<T, DP> F;
    constexpr int kSub = F::kSub, kKey = F::kKey, kVBytes = F::kVBytes, kChunks = F::kChunks, kEach = F::kEach, BN = 16 * kSub;
    constexpr int kStride = DP + 4, kWords = kVBytes / 4;
    constexpr bool kBf16 = sizeof(T) == 2;
    float *const sums = shared.sums;
    float2(*const stats)[16] = shared.stats;
    const int lane = threadIdx.x & 63, quarter = lane >> 4, mine = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t bytes = a.dim * (int32_t)sizeof(T);
    Work w;
    if (!find_work<16, 16, MODE>(a, piece, mine, 0, item, w)) return;
    const int32_t lo_at = w.lo, hi_at = w.hi;
    const Keys keys = keys_of(a, w, lo_at, hi_at, BN, part, piece.parts, piece.least);
    const int32_t at = w.valid ? w.at : -1;
    const int32_t first = keys.first + (WAVES > 1 ? wave : 0), last_page = keys.n > 0 ? (keys.n - 1) >> a.page_shift : 0;
    // pages of a tile's tokens: of its sixteens, or of a token a lane; looked up a tile ahead
    struct Pages {
        int32_t page[BYPAGE ? kSub : 1];
    };
    auto find_pages = [&](int32_t base) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int i = 0; i < (BYPAGE ? kSub : 1); ++i) {
            const int32_t x = (BYPAGE ? base + 16 * i : base + (lane & (BN - 1))) >> a.page_shift, there = x < last_page ? x : last_page;
            p.page[i] = BYPAGE ? scalar_load(w.table + there) : w.table[there];
        }
        return p;
    };
    // (behind the wave's last tile that one again: what is loaded in advance is then of no use, but there)
    auto tile_base = [&](int32_t t) __attribute__((always_inline)) { return keys.base(t < keys.last ? t : keys.last - 1 - (keys.last - 1 - first) % WAVES, BN); };
    Pages ahead;
    if (first < keys.last) ahead = find_pages(keys.base(first, BN));

    // the queries, zeros where there is none and past the row's end
    u32x4 q[kKey];
    {
        const char *const from = (const char *)a.q + (w.token * a.ldq + (int64_t)w.qhead * a.dim) * (int64_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < kKey; ++i) {
            const int32_t o = (i * 4 + quarter) * 16;
            q[i] = u32x4{0, 0, 0, 0};
            if (w.valid && a.scale != 0.f && (FULL || o < bytes)) q[i] = *reinterpret_cast<const u32x4_any *>(from + o);
            if (a.scale < 0.f) q[i] ^= kBf16 ? 0x80008000u : 0x80000000u;
        }
    }
    const float scale = weight_scale(a);
    f32x4 o[kChunks][kEach];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < kEach; ++e) o[c][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, l = 0.f;
    bool odd = false;

    const int32_t slots = (1 << a.page_shift) - 1;
    const char *const keys_at = (const char *)a.k + ((int64_t)w.head << a.page_shift) * bytes;
    const int64_t values_behind = (const char *)a.v - (const char *)a.k;
    u32x4 k[kSub][kKey];
    uint32_t v[kSub * 4][kChunks][kWords];
    // where the rows of a tile's tokens are
    struct Rows {
        const char *row16[BYPAGE ? kSub : 1];
        int32_t base, page;
    };
    auto rows_at = [&](int32_t base, Pages now) __attribute__((always_inline)) {
        Rows at;
        at.base = base;
#pragma unroll
        for (int i = 0; i < (BYPAGE ? kSub : 1); ++i) {
            now.page[i] = now.page[i] < 0 ? 0 : now.page[i];
            now.page[i] = now.page[i] < a.pages ? now.page[i] : a.pages - 1;
            at.row16[i] = keys_at + (uint64_t)(uint32_t)now.page[i] * a.page_bytes + (uint32_t)(((base + 16 * i) & slots) * bytes);
        }
        at.page = now.page[0];
        return at;
    };
    // (rows past the last key are of its page, or the last key's: theirs is taken by nobody)
    auto row_of = [&](const Rows &at, int s, int x) __attribute__((always_inline)) -> const char * {
        if constexpr (BYPAGE) return at.row16[s] + x * bytes;
        const int32_t page = __shfl(at.page, 16 * s + x, kWave), token = at.base + 16 * s + x;
        return keys_at + (uint64_t)(uint32_t)page * a.page_bytes + (uint32_t)(((token < keys.n ? token : keys.n - 1) & slots) * bytes);
    };
    // (past a row's end its first piece stands in: of keys it is made zeros before the product, since the queries' zeros are not enough
    // where it holds an infinity; what comes out of the values is not stored)
    auto load_keys = [&](const Rows &at) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < kSub; ++s) {
            const char *const row = row_of(at, s, mine);
#pragma unroll
            for (int i = 0; i < kKey; ++i) {
                const int32_t at_byte = (i * 4 + quarter) * 16;
                k[s][i] = *reinterpret_cast<const u32x4 *>(row + (FULL || at_byte < bytes ? at_byte : 0));
            }
        }
    };
    auto load_values = [&](const Rows &at) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kSub * 4; ++e) {
            const char *const row = row_of(at, e >> 2, quarter * 4 + (e & 3)) + values_behind;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int32_t at_byte = (c * 16 + mine) * kVBytes;
                const char *const p = row + (FULL || at_byte < bytes ? at_byte : 0);
                if constexpr (kVBytes == 8) {
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
                    v[e][c][0] = x[0];
                    v[e][c][1] = x[1];
                } else {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[e][c][i] = x[i];
                }
            }
        }
    };
    if (first < keys.last) {
        const Rows at = rows_at(keys.base(first, BN), ahead);
        ahead = find_pages(tile_base(first + WAVES));
        load_keys(at);
        load_values(at);
    }
#pragma unroll 1
    for (int32_t t = first; t < keys.last; t += WAVES) {
        const int32_t base = keys.base(t, BN);
        // scores
        f32x4 s4[kSub];
#pragma unroll
        for (int s = 0; s < kSub; ++s) {
            s4[s] = f32x4{0.f, 0.f, 0.f, 0.f};
            // fp32: four sums, which stay smaller than one, and so their roundings (256 dimensions: errors against 64 bits 1.0e-6 in one
            // sum, below 6e-7 in four; the same time)
            f32x4 chains[4] = {s4[s], s4[s], s4[s], s4[s]};
#pragma unroll
            for (int i = 0; i < kKey; ++i) {
                if (!FULL && (i * 4 + 3) * 16 >= kLeastDim<T, DP> * (int)sizeof(T) && (i * 4 + quarter) * 16 >= bytes) k[s][i] = u32x4{0, 0, 0, 0};
                if constexpr (kBf16) {
                    s4[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s][i]), __builtin_bit_cast(bf16x8, q[i]), s4[s], 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        chains[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)k[s][i][e]),
                                                                         __builtin_bit_cast(float, (uint32_t)q[i][e]), chains[e], 0, 0, 0);
                }
            }
            if constexpr (!kBf16) s4[s] = (chains[0] + chains[1]) + (chains[2] + chains[3]);
        }
        // the next tile's keys take their registers, and its values theirs behind this tile's
        const Rows next = rows_at(tile_base(t + WAVES), ahead);
        ahead = find_pages(tile_base(t + 2 * WAVES));
        load_keys(next);
        float p[kSub * 4];
#pragma unroll
        for (int e = 0; e < kSub * 4; ++e) p[e] = s4[e >> 2][e & 3];
        if (!keys.whole(base, BN)) {
            uint32_t largest = 0;
#pragma unroll
            for (int e = 0; e < kSub * 4; ++e) {
                const int32_t x = base + 16 * (e >> 2) + quarter * 4 + (e & 3);
                p[e] = keys.seen(x, at) ? p[e] : kNone;
                // what no query sees may be anything, and 0 * NaN is NaN
                const uint32_t keep = keys.seen_by_some(x) ? 0xffffffffu : 0u;
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        v[e][c][i] &= keep;
                        largest = larger_magnitude<T>(largest, v[e][c][i]);
                    }
            }
            // A value that is no number, seen by some queries and not by others of the tile: it is left out of the product, and
            // added to those that see it at the end.
            if (MODE != kAttendOwn && lo_at != hi_at && __any(no_number<T>(largest))) {
                odd = true;
#pragma unroll
                for (int e = 0; e < kSub * 4; ++e)
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int i = 0; i < kWords; ++i) v[e][c][i] = numbers<T>(v[e][c][i]);
            }
        }
        // the running maximum, the same in the four lanes of a query
        float top = p[0];
#pragma unroll
        for (int e = 1; e < kSub * 4; ++e) top = fmaxf(top, p[e]);
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        if (__any(top > m)) {
            const float now = fmaxf(top, m);
            const float by = now == kNone ? 1.f : __builtin_amdgcn_exp2f((m - now) * scale);
            m = now;
            l *= by;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int e = 0; e < kEach; ++e) o[c][e] *= by;
        }
        const float ref = m == kNone ? 0.f : m;
#pragma unroll
        for (int e = 0; e < kSub * 4; ++e) p[e] = __builtin_amdgcn_exp2f((p[e] - ref) * scale);
        if constexpr (kBf16) {
            // Weights go into the product as bf16; l adds up the rounded ones, so that they come to 1 all the same.
            u32x4 pw;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pw[i] = weights2(p[2 * i], p[2 * i + 1]);
                l += __builtin_bit_cast(float, (uint32_t)pw[i] << 16) + __builtin_bit_cast(float, (uint32_t)pw[i] & 0xffff0000u);
            }
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    u32x4 vw;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        vw[i] = __builtin_amdgcn_perm(v[2 * i + 1][c][e >> 1], v[2 * i][c][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
                    o[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw), __builtin_bit_cast(bf16x8, pw), o[c][e], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                l += p[j];
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int e = 0; e < kEach; ++e)
                        o[c][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v[j][c][e]), p[j], o[c][e], 0, 0, 0);
            }
        }
        load_values(next);
    }

    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (l != l && m == kNone) m = 0.f;                 // (a query that is no number: its maximum says nothing, its sum does)
    if constexpr (WAVES == 1) {
        // a lane has kEach values after each other of its query
        if (!w.valid) return;
        const int64_t row = w.token * a.heads + w.qhead, at_part = row * a.parts + piece.part0 + part;
        const float by = a.parts > 1 ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;
        if (a.parts > 1 && quarter == 0) a.stats[at_part] = float2{m, l};
        if (a.parts > 1 && m == kNone) return;
        T *const out = (T *)a.out + w.token * a.ldo + (int64_t)w.qhead * a.dim;
        float *const sums_out = a.sums + at_part * a.dim;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t d = (c * 16 + quarter * 4 + r) * kEach;
                if (!FULL && d >= a.dim) continue;
                float y[kEach];
#pragma unroll
                for (int e = 0; e < kEach; ++e) y[e] = o[c][e][r] * by;
                if (a.parts > 1) store_some(sums_out + d, y);
                else store_some(out + d, y);
            }
        return;
    }
    // the four waves' parts
    if (quarter == 0) stats[wave][mine] = float2{m, l};
    if (threadIdx.x < 16) {
        shared.token[mine] = w.valid ? w.token : -1;
        shared.head[mine] = w.qhead;
    }
    __syncthreads();
    float M = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i) M = fmaxf(M, stats[i][mine].x);
    const float by = m == kNone ? 0.f : __builtin_amdgcn_exp2f((m - M) * scale);
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float *const to = sums + (wave * 16 + mine) * kStride + (c * 16 + quarter * 4 + r) * kEach;
#pragma unroll
            for (int e = 0; e < kEach; e += 2) *reinterpret_cast<f32x2 *>(to + e) = f32x2{o[c][e][r] * by, o[c][e + 1][r] * by};
        }
    if (MODE != kAttendOwn && odd) add_odd_values<T, 16>(a, w, keys, BN, wave, 4, at, sums + wave * 16 * kStride, kStride, 0, a.dim);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (DP / 8); i += 256) {
        const int r = i / (DP / 8), d = i % (DP / 8) * 8;
        if (d >= a.dim) continue;
        const int64_t token = shared.token[r];
        const int32_t head = shared.head[r];
        if (token < 0) continue;
        float top = kNone, total = 0.f, y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, stats[j][r].x);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (stats[j][r].x != kNone) total += stats[j][r].y * __builtin_amdgcn_exp2f((stats[j][r].x - top) * scale);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += sums[(j * 16 + r) * kStride + d + e];
        if (a.parts == 1) {
            const float inverse = total > 0.f || total != total ? 1.f / total : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= inverse;
            store8((T *)a.out + token * a.ldo + (int64_t)head * a.dim + d, y);
        } else {
            const int64_t at_part = (token * a.heads + head) * a.parts + piece.part0 + part;
            if (d == 0) a.stats[at_part] = float2{top, total};
            if (top != kNone) store8(a.sums + at_part * a.dim + d, y);
        }
    }
}

// ---------------------------------------------------------------- 128 queries a block, keys through LDS

// Where many queries share a key head (a prompt's rows, a prompt's own tokens) the matrix instructions bound it, and the rate
// at which operands reach them: four waves of 32 queries each share tiles of 64 keys (32 of 256 dimensions), which go from memory to LDS
// without registers, the next tile's while this one is worked on.  As above both products are transposed,
// on v_mfma_f32_32x32x16_bf16: S^T = K Q^T leaves register v of lane l the score of token 8 (v / 4) + 4 (l / 32) + v % 4 of 32 for query
// l % 32; so a lane's P^T for 16 tokens is its registers 8 i .. 8 i + 7 in pairs, and V^T is read from LDS transposed
// (ds_read_b64_tr_b16: of 16 lanes that read 4 rows of 16 values, each gets one column) for the same tokens.
// In LDS a row's 16-byte pieces are exchanged (by its number, piece c at c ^ f(row)), so that neither the rows that 16 lanes
// read of K nor the four rows they read of V meet in a bank.
// A query's reference m is raised only when a score passes it by 2^8: weights up to 256 are as good as weights up to 1.
// Bound by the matrix pipes and the clock that their power leaves: 8192 tokens, 32 heads of 128 over 8, causal, 510 to 527 us from card to
// card = 1.04 to 1.08 PFLOP/s, pipes busy 54 % of the cycles (a library product of 8192^3 has 1.37).  On the way: 625 us with the
// compiler's own requests, which it waited for before each read of LDS; 575 by hand; 542 with the next tile's products under this
// tile's exponentials; 522 with the waves' products put before other waves' work and fewer scalar instructions a tile; 515 with
// maxima of products in place of scores.
template <int DP> struct TileForm {
    static constexpr int kKeys = DP == 256 ? 32 : 64, kPieces = DP / 8, kBytes = kKeys * DP * 2, kLoads = kBytes / 4096, kRowsEach = 64 / kPieces;
    static constexpr int kQueries = 128, kStride = 68;
    static constexpr int kLds = 4 * kBytes > kQueries * kStride * 4 ? 4 * kBytes : kQueries * kStride * 4;
    static __device__ __forceinline__ int key_place(int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int value_place(int row) { return DP == 64 ? (row >> 1 & 1) << 2 : (row & 3) << 2; }
};

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

// 16 bytes a lane from memory to LDS, lane after lane from `to` on (the same for the wave).  By hand, since the compiler would wait
// for the tile that is on its way before each read of the one that is there: it takes them for one memory.  The instruction
// writes no register; its end is waited for at the top of the loop over tiles, and what the compiler itself counts can only
// come out as a longer wait.
template <int N>                  // N KiB, each a KiB behind the one before both there and here
__device__ __forceinline__ void fetch_lds(const char *base, const int32_t (&offset)[N], unsigned char *to)
{
    static_assert(N == 1 || N == 2 || N == 4, "written out for these");
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void *)to);
    const uint64_t low = (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(uintptr_t)base),
                   high = (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)((uintptr_t)base >> 32));
    base = (const char *)(low | high << 32);
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1" ::"s"(at), "s"(base), "v"(offset[0]) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024" ::"s"(at),
                     "s"(base), "v"(offset[0]), "v"(offset[1])
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:%6\n\t"
                     "global_load_lds_dwordx4 %4, %1 offset:%7\n\tglobal_load_lds_dwordx4 %5, %1 offset:%8" ::"s"(at),
                     "s"(base), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "n"(1 << 10), "n"(2 << 10), "n"(3 << 10)
                     : "memory");
}
__device__ __forceinline__ void fetch_lds(const char *from, unsigned char *to)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from) : "memory");
}
// What the wave has asked for has landed, what it has read of LDS is there, and so with the block's other waves.
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ const u32x4 kZeros = {0, 0, 0, 0};             // what stands in for keys past a row's end

template <int DP> struct TilesShared {
    __attribute__((aligned(1024))) unsigned char smem[TileForm<DP>::kLds];
    int64_t token[TileForm<DP>::kQueries];             // of each query, -1: none ...
    int32_t head[TileForm<DP>::kQueries];              // ... and its head
    int32_t any_odd;
};

// The other half of a wave's value beside a lane's own.
__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

template <int DP, bool FULL, bool BYPAGE, int MODE>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, const AttendPiece &piece, uint32_t item, int32_t part, TilesShared<DP> &shared)
{
    typedef TileForm<DP> F;
    constexpr int BN = F::kKeys, kLoads = F::kLoads, kPieces = F::kPieces, kStride = F::kStride, kRow = DP * 2;
    unsigned char *const smem = shared.smem;
    int32_t &any_odd = shared.any_odd;
    const int lane = threadIdx.x & 63, half = lane >> 5, mine = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t bytes = a.dim * 2;
    Work w;
    if (!find_work<F::kQueries, 32, MODE>(a, piece, wave * 32 + mine, wave * 32, item, w)) return;
    const int32_t at = w.valid ? w.at : -1;
    if (lane < 32) {
        shared.token[wave * 32 + mine] = w.valid ? w.token : -1;
        shared.head[wave * 32 + mine] = w.qhead;
    }
    if (threadIdx.x == 0) any_odd = 0;
    const int32_t lo = w.lo, hi = w.hi, wave_lo = w.wave_lo, wave_hi = w.wave_hi;
    // the queries (zeros where there is none and past the row's end)
    u32x4 q[DP / 16];
    {
        const char *const from = (const char *)a.q + (w.token * a.ldq + (int64_t)w.qhead * a.dim) * 2;
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int32_t o = (i * 2 + half) * 16;
            q[i] = u32x4{0, 0, 0, 0};
            if (w.valid && a.scale != 0.f && (FULL || o < bytes)) q[i] = *reinterpret_cast<const u32x4_any *>(from + o);
            q[i] ^= sign;
        }
    }
    const float scale = weight_scale(a);
    const Keys keys = keys_of(a, w, lo, hi, BN, part, piece.parts, piece.least);

    // What a wave fetches of a tile: BN / 4 rows after each other (all in one page, of pages of 16 tokens and more), kLoads KiB, of which
    // a lane takes 16 bytes each, such that they land in their place.
    constexpr int kWaveRows = BN / 4;
    const int32_t row0 = wave * kWaveRows + lane / kPieces;           // (load i: i kRowsEach further on)
    constexpr int kValueOffs = F::kRowsEach % 4 == 0 ? 1 : kLoads;        // (where a load's rows start the exchange anew, one for all)
    int32_t key_off[kLoads], value_off[kValueOffs];
    const int32_t in_rows = BYPAGE ? lane / kPieces * bytes : 0;
    // (past a row's end zeros from elsewhere stand in for keys, below 0 here: the queries' own would not do where what stands in holds
    // an infinity; and the row's first piece for values: what comes out of them there is not stored.  2 chunks of up to 1072 queries, 16
    // heads of 168 on one: 58.0 us with the row's first piece for keys too, 58.7 so, 61 with zeros put in as keys are read from LDS, 64.5
    // with those lanes' requests left out; 6 of up to 362, 40 heads of 80, window 23: 24.9, 26.6, 26.7, 31.3)
    auto piece_of = [&](int place, int32_t stand_in) __attribute__((always_inline)) {
        const int32_t at_byte = ((lane % kPieces) ^ place) * 16;
        return FULL || at_byte < bytes ? in_rows + at_byte : stand_in;
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) key_off[i] = piece_of(F::key_place(row0 + i * F::kRowsEach), -1);
#pragma unroll
    for (int i = 0; i < kValueOffs; ++i) value_off[i] = piece_of(F::value_place(row0 + i * F::kRowsEach), in_rows);
    const int32_t last_page = keys.n > 0 ? (keys.n - 1) >> a.page_shift : 0, slots = (1 << a.page_shift) - 1;
    const char *const keys_at = (const char *)a.k + ((int64_t)w.head << a.page_shift) * bytes;
    const char *const values_at = (const char *)a.v + ((int64_t)w.head << a.page_shift) * bytes;
    struct Pages {
        int32_t page[BYPAGE ? 1 : kLoads];
    };
    auto find_pages = [&](int32_t base) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int i = 0; i < (BYPAGE ? 1 : kLoads); ++i) {
            const int32_t x = (base + (BYPAGE ? wave * kWaveRows : row0 + i * F::kRowsEach)) >> a.page_shift;
            if constexpr (BYPAGE) p.page[i] = scalar_load(w.table + (x < last_page ? x : last_page));
            else p.page[i] = w.table[x < last_page ? x : last_page];
        }
        return p;
    };
    // keys (to LDS buffer 0 or 1) or values (2 or 3) of the tile
    auto fetch = [&](int32_t base, const Pages &p, int buffer) __attribute__((always_inline)) {
        unsigned char *const to = smem + buffer * F::kBytes + wave * (kWaveRows * kRow);
        const char *const from = buffer < 2 ? keys_at : values_at;
        auto off = [&](int i) __attribute__((always_inline)) { return buffer < 2 ? key_off[i] : value_off[i % kValueOffs]; };
        if constexpr (BYPAGE) {
            int32_t page = p.page[0] < 0 ? 0 : p.page[0];
            page = page < a.pages ? page : a.pages - 1;
            const char *const at = from + ((uint64_t)(uint32_t)page * a.page_bytes + (uint32_t)(((base + wave * kWaveRows) & slots) * bytes));
            if constexpr (FULL) {
                // (load i's KiB lies i KiB behind the first both in memory and in LDS, which the instruction adds)
                int32_t offs[kLoads];
#pragma unroll
                for (int i = 0; i < kLoads; ++i) offs[i] = off(i);
                fetch_lds(at, offs, to);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    if (buffer < 2) fetch_lds(off(i) < 0 ? (const char *)&kZeros : at + (i * F::kRowsEach * bytes + off(i)), to + i * 1024);
                    else fetch_lds(at + i * F::kRowsEach * bytes, {off(i)}, to + i * 1024);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int32_t x = base + row0 + i * F::kRowsEach, there = x < keys.n ? x : keys.n - 1;
                int32_t page = p.page[i] < 0 ? 0 : p.page[i];
                page = page < a.pages ? page : a.pages - 1;
                const char *const at = from + ((uint64_t)(uint32_t)page * a.page_bytes + (uint32_t)((there & slots) * bytes + off(i)));
                fetch_lds(!FULL && off(i) < 0 ? (const char *)&kZeros : at, to + i * 1024);
            }
        }
    };

    f32x16 o[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m = kNone, l = 0.f;
    // A weight by one instruction less, 2^(s scale - ref), ref = m scale rounded, where the rounding is far from mattering: sums are then
    // relative to 2^ref, and `rest` is what m scale is beyond it, for where they meet others.
    constexpr float kFar = 1 << 16;
    const float slack = fminf(8.f / scale, 0x1.fffffep127f);
    auto rest = [&](float x) __attribute__((always_inline)) {
        const float ref = x * scale;
        return fabsf(ref) < kFar ? fmaf(x, scale, -ref) : 0.f;
    };
    typedef f32x16 Scores[BN / 32];
    const int kx = (half ^ F::key_place(mine)) * 16;
    const int32_t vrow = 4 * half + (lane & 15) / 4;
    // a tile that every query of the wave sees whole, of the block
    const int32_t wave_whole = (keys.n < wave_lo + 1 ? keys.n : wave_lo + 1) - BN, block_whole = (keys.n < lo + 1 ? keys.n : lo + 1) - BN;
    const int32_t wave_from = a.window > 0 ? wave_hi - a.window : -1, block_from = a.window > 0 ? hi - a.window : -1;

    // The pieces of a tile's work, in the order that they are to be issued in: the products of scores a key fragment ahead of
    // their operands, with a share of another tile's weights under each.
    constexpr int kScoreSteps = BN / 32 * (DP / 16), kValueSteps = BN / 16 * (DP / 32), kPairs = BN / 4;
    auto key_fragment = [&](const unsigned char *krow, int j) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8 *>(krow + j % (BN / 32) * 32 * kRow + ((j / (BN / 32) * 32) ^ kx));
    };
    auto value_fragment = [&](const unsigned char *vrows, int j) __attribute__((always_inline)) {
        const int i = j / (DP / 32), d = j % (DP / 32), c = (d * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ F::value_place(vrow);
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(vrows + i * 16 * kRow + c * 16));
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(vrows + (i * 16 + 8) * kRow + c * 16));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // two of a lane's weights, rounded to bf16 for the second product; l adds up the rounded ones, so that they come to 1 all the same
    auto weigh = [&](const Scores &s, int j, float ref) __attribute__((always_inline)) -> uint32_t {
        const float x = s[j >> 3][j % 8 * 2], y = s[j >> 3][j % 8 * 2 + 1];
        const uint32_t w2 = weights2(__builtin_amdgcn_exp2f(fmaf(x, scale, -ref)), __builtin_amdgcn_exp2f(fmaf(y, scale, -ref)));
        l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w2), __builtin_bit_cast(bf16x2, 0x3f803f80u), l, false);
        return w2;
    };
    auto score = [&](const unsigned char *ks, Scores &s, auto under) __attribute__((always_inline)) {
        const unsigned char *const krow = ks + mine * kRow;
        bf16x8 k[3] = {key_fragment(krow, 0), key_fragment(krow, 1), key_fragment(krow, 2)};
#pragma unroll
        for (int j = 0; j < kScoreSteps; ++j) {
            const int b = j % (BN / 32), i = j / (BN / 32);
            if (i == 0) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
            }
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[j % 3], __builtin_bit_cast(bf16x8, q[i]), s[b], 0, 0, 0);
            if (j + 3 < kScoreSteps) k[j % 3] = key_fragment(krow, j + 3);
            under(j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto hide = [&](int32_t base, Scores &s) __attribute__((always_inline)) {
        if (base <= wave_whole && (base > wave_from || base + BN <= keys.sinks)) return;
        const int32_t first = base + 4 * half, upto = (at < keys.n ? at : keys.n - 1) - first;      // (of the tile's tokens, as the lane has them)
        if (a.window > 0) {
            // (unsigned, since a query before the tile's first may pass -2^31 here: it sees none of it whatever comes out)
            const int32_t from = (int32_t)((uint32_t)at - (uint32_t)a.window - (uint32_t)first), sinks = keys.sinks - first;
#pragma unroll
            for (int b = 0; b < BN / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int x = b * 32 + 8 * (r >> 2) + (r & 3);
                    const float y = x < sinks ? s[b][r] : kNone, z = x > from ? s[b][r] : y;
                    s[b][r] = x <= upto ? z : kNone;
                }
        } else {
#pragma unroll
            for (int b = 0; b < BN / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + 8 * (r >> 2) + (r & 3) <= upto ? s[b][r] : kNone;
        }
    };
    auto add_values = [&](const unsigned char *vs, const u32x4 (&pw)[BN / 16]) __attribute__((always_inline)) {
        const unsigned char *const vrows = vs + vrow * kRow + (lane & 1) * 8;
        bf16x8 v[3] = {value_fragment(vrows, 0), value_fragment(vrows, 1), value_fragment(vrows, 2)};
#pragma unroll
        for (int j = 0; j < kValueSteps; ++j) {
            const int i = j / (DP / 32), d = j % (DP / 32);
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[j % 3], __builtin_bit_cast(bf16x8, pw[i]), o[d], 0, 0, 0);
            if (j + 3 < kValueSteps) v[j % 3] = value_fragment(vrows, j + 3);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One tile: its weights and their product with its values, under it the next tile's scores; the tile after that one's keys and
    // the next one's values are asked for.
    Pages next_pages, after_pages;                     // of the next tile and the one after it (a page a lane: looked up a step before)
    auto pages_of = [&](int32_t t) __attribute__((always_inline)) { return find_pages(keys.base(t < keys.last ? t : keys.last - 1, BN)); };
    auto step = [&](int32_t t, int32_t base, int buffer, Scores &now, Scores &next) __attribute__((always_inline)) {
        tile_barrier();
        const bool more = t + 1 < keys.last;
        const int32_t next_base = keys.base(t + 1, BN);
        if (more) fetch(next_base, next_pages, 2 + (buffer ^ 1));
        if (t + 2 < keys.last) {
            const int32_t after_base = keys.base(t + 2, BN);
            if constexpr (BYPAGE) after_pages = find_pages(after_base);        // (by the scalar cache)
            fetch(after_base, after_pages, buffer);
        }
        next_pages = after_pages;
        if constexpr (!BYPAGE) after_pages = pages_of(t + 3);
        unsigned char *const vs = smem + (2 + buffer) * F::kBytes;
        if (!(base <= block_whole && (base > block_from || base + BN <= keys.sinks))) {
            // what no query sees may be anything, and 0 * NaN is NaN; what is no number and seen by some alone is added at the end
            for (int i = threadIdx.x; i < BN * kPieces; i += 256) {
                u32x4 *const p = reinterpret_cast<u32x4 *>(vs) + i;
                if (!keys.seen_by_some(base + i / kPieces)) *p = u32x4{0, 0, 0, 0};
                else if (lo != hi) {
                    u32x4 x = *p;
                    uint32_t largest = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) largest = larger_magnitude<uint16_t>(largest, x[e]);
                    if (no_number<uint16_t>(largest)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = numbers<uint16_t>(x[e]);
                        *p = x;
                        any_odd = 1;
                    }
                }
            }
            __syncthreads();
        }
        if (wave_hi < 0) return;                       // (no queries)
        float top = kNone;
#pragma unroll
        for (int b = 0; b < BN / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, now[b][r]);
        top = halves_max(top);
        if (__any(top > m + slack)) {
            // (each query by its own scores alone: what a neighbour asks for is not to change its bits)
            const bool raised = top > m + slack;
            const float by = raised ? __builtin_amdgcn_exp2f(fmaf(m - top, scale, rest(top) - rest(m))) : 1.f;
            m = raised ? top : m;
            l *= by;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) o[i] *= by;
        }
        float ref = m == kNone ? 0.f : m * scale;
        const bool far = fabsf(ref) >= kFar;
        if (__any(far)) {
            ref = far ? 0.f : ref;
#pragma unroll
            for (int b = 0; b < BN / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) now[b][r] = far ? now[b][r] - m : now[b][r];
        }
        u32x4 pw[BN / 16];
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        if (more) {
            score(smem + (buffer ^ 1) * F::kBytes, next, [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int e = j * kPairs / kScoreSteps; e < (j + 1) * kPairs / kScoreSteps; ++e) pw[e / 4][e % 4] = weigh(now, e, ref);
            });
        } else {
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                pw[e / 4][e % 4] = weigh(now, e, ref);
                if (e % 2) __builtin_amdgcn_sched_barrier(0);
            }
        }
        add_values(vs, pw);
        __builtin_amdgcn_s_setprio(0);
        if (more) hide(next_base, next);
    };
    if (keys.first < keys.last) {
        const int32_t base = keys.base(keys.first, BN);
        const Pages pages = find_pages(base);
        next_pages = pages_of(keys.first + 1);
        if constexpr (!BYPAGE) after_pages = pages_of(keys.first + 2);
        fetch(base, pages, 0);
        fetch(base, pages, 2);
        tile_barrier();
        if (keys.first + 1 < keys.last) fetch(keys.base(keys.first + 1, BN), next_pages, 1);
        Scores one, two;
        score(smem, one, [](int) {});
        hide(base, one);
        int32_t t = keys.first;
#pragma unroll 1
        for (;;) {
            step(t, keys.base(t, BN), 0, one, two);
            if (++t >= keys.last) break;
            step(t, keys.base(t, BN), 1, two, one);
            if (++t >= keys.last) break;
        }
    }

    // sums to memory, 64 dimensions of a wave's queries at a time through its part of LDS
    l += __shfl_xor(l, 32, kWave);
    if (l != l && m == kNone) m = 0.f;
    const float by = a.parts > 1 ? __builtin_amdgcn_exp2f(-rest(m)) : l > 0.f || l != l ? 1.f / l : 0.f;
    l *= by;
    __syncthreads();
    const bool odd = any_odd != 0;
    float *const sums = reinterpret_cast<float *>(smem) + wave * 32 * kStride;
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
        if (c * 64 >= a.dim) break;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = o[c * 2 + i][r + e] * by;
                *reinterpret_cast<f32x4 *>(sums + mine * kStride + i * 32 + 2 * r + 4 * half) = x;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        if (odd) add_odd_values<uint16_t, 32>(a, w, keys, BN, 0, 1, at, sums, kStride, c * 64, c * 64 + 64 < a.dim ? c * 64 + 64 : a.dim);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + lane / 8, d = c * 64 + lane % 8 * 8;
            const int64_t token = shared.token[wave * 32 + r];
            const int32_t head = shared.head[wave * 32 + r];
            const float ml = __shfl(m, r, kWave), ll = __shfl(l, r, kWave);
            if (token < 0 || d >= a.dim) continue;
            float y[8];
            const float *const from = sums + r * kStride + lane % 8 * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = from[e];
            if (a.parts == 1) {
                store8((uint16_t *)a.out + token * a.ldo + (int64_t)head * a.dim + d, y);
            } else {
                const int64_t at_part = (token * a.heads + head) * a.parts + piece.part0 + part;
                if (d == 0) a.stats[at_part] = float2{ml, ll};
                if (ml != kNone) store8(a.sums + at_part * a.dim + d, y);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------- launches of both

// Which work is block b's: of a piece's items, of which `tiles` after each other read the same keys, those of a group go to one
// XCD (blocks go round the eight), whose L2 then has the keys; of ragged queries the last first, which see most keys.
template <int MODE> __device__ __forceinline__ void item_of(const AttendPiece &p, uint32_t b, uint32_t *item, int32_t *part)
{
    if (p.parts == 1 && p.tiles == 1) {
        *part = 0;
        *item = MODE == kAttendRagged ? p.blocks - 1 - b : b;
        return;
    }
    if constexpr (MODE == kAttendRagged) {
        const uint32_t x = b / p.blocks;
        *part = (int32_t)x;
        *item = p.blocks - 1 - (b - x * p.blocks);
        return;
    }
    const uint32_t tiles = p.tiles, groups = p.groups, whole = (groups * p.parts & ~7u) * tiles;
    uint32_t group, tile;
    if (b < whole) {
        const uint32_t j = b >> 3, g = j / tiles;
        tile = j - g * tiles;
        group = g * 8 + (b & 7);
    } else {
        group = b / tiles;
        tile = b - group * tiles;
    }
    const uint32_t x = group / groups;
    *part = (int32_t)x;
    *item = (group - x * groups) * tiles + tile;
}

// With two pieces (what rows share, and their own) every `every`-th block is one of the first, as long as there are any.
__device__ __forceinline__ bool first_piece(const AttendPieces &p, uint32_t *b)
{
    if (p.count < 2) return true;
    const uint32_t all = p.piece[0].blocks * p.piece[0].parts, turn = *b / p.every;
    if (turn < all && *b == turn * p.every) {
        *b = turn;
        return true;
    }
    *b -= turn < all ? turn + 1 : all;
    return false;
}

// A block's share of rows' own tokens.
template <class T, int DP, bool FULL, bool BYPAGE>
__device__ __forceinline__ void attend_own(const AttendArgs &a, const AttendPiece &piece, uint32_t b, RowsShared<T, DP> &shared)
{
    uint32_t item;
    int32_t part;
    if (piece.alone) {
        item = b * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (item < piece.items) attend_rows<T, DP, FULL, BYPAGE, 1, kAttendOwn>(a, piece, item, 0, shared);
        return;
    }
    item_of<kAttendOwn>(piece, b, &item, &part);
    attend_rows<T, DP, FULL, BYPAGE, 4, kAttendOwn>(a, piece, item, part, shared);
}

template <class T, int DP, bool FULL, bool BYPAGE>
__global__ __launch_bounds__(256, DP == 96 ? 3 : 1) void attend_own_kernel(AttendArgs a, AttendPieces p)
{
    __shared__ RowsShared<T, DP> shared;
    attend_own<T, DP, FULL, BYPAGE>(a, p.piece[0], blockIdx.x, shared);
}

// Queries of prompts, or of rows that share a prompt (MODE) with what is the rows' own beside them: 16 a block, or 128.
// (fp32 rows of up to 96 dimensions: three blocks a compute unit, for which the compiler has to save a few registers: nine chunks of up
// to 301 tokens behind up to 77, 6 heads of 72 over 2, 29.1 us with two, 24.5 with three)
template <class T, int DP, bool FULL, bool BYPAGE, int MODE>
__global__ __launch_bounds__(256, DP == 96 ? 3 : 1) void attend_rows_kernel(AttendArgs a, AttendPieces p)
{
    __shared__ RowsShared<T, DP> shared;
    uint32_t b = blockIdx.x, item;
    int32_t part;
    if (MODE == kAttendRagged || first_piece(p, &b)) {
        item_of<MODE>(p.piece[0], b, &item, &part);
        attend_rows<T, DP, FULL, BYPAGE, 4, MODE>(a, p.piece[0], item, part, shared);
    } else if constexpr (MODE != kAttendRagged) {
        attend_own<T, DP, FULL, BYPAGE>(a, p.piece[1], b, shared);
    }
}

template <int DP, bool FULL, bool BYPAGE, int MODE>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attend_tiles_kernel(AttendArgs a, AttendPieces p)
{
    __shared__ union Shared {
        TilesShared<DP> tiles;
        RowsShared<uint16_t, DP> rows;
    } shared;
    uint32_t b = blockIdx.x, item;
    int32_t part;
    if (MODE == kAttendRagged || first_piece(p, &b)) {
        item_of<MODE>(p.piece[0], b, &item, &part);
        attend_tiles<DP, FULL, BYPAGE, MODE>(a, p.piece[0], item, part, shared.tiles);
    } else if constexpr (MODE != kAttendRagged) {
        attend_own<uint16_t, DP, FULL, BYPAGE>(a, p.piece[1], b, shared.rows);
    }
}

// ---------------------------------------------------------------- parts joined

// A wave a query head: the parts' m and l a lane each, then their sums a part after the other.  Bound by the memory (1024 rows of 32
// heads of 128 in three parts: 17 us, 52 MB); a launch of its own, 4 us where there is little to do.
template <class T>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    const int lane = threadIdx.x & 63;
    const uint32_t i = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t token = i / (uint32_t)a.heads;       // (the launch sees to it that they fit)
    if (token >= a.tokens) return;
    if (a.offsets) {
        if (token < offset_at(a, 0) || token >= offset_at(a, a.rows)) return;
        if (a.finished && a.finished[find_sequence<0>(a, token, 1).s]) return;
    } else if (a.finished && a.finished[token]) return;
    const float2 *const stats = a.stats + (int64_t)i * a.parts;
    const float2 mine = lane < a.parts ? stats[lane] : float2{kNone, 0.f};
    const float M = wave_max(mine.x);
    const float weight = mine.x == kNone ? 0.f : __builtin_amdgcn_exp2f((mine.x - M) * weight_scale(a));
    const float total = wave_sum(weight * mine.y);
    const float inverse = total > 0.f || total != total ? 1.f / total : 0.f;
    const uint64_t there = __ballot(mine.x != kNone);
    const float *const sums = a.sums + (int64_t)i * a.parts * a.dim;
    T *const out = (T *)a.out + token * a.ldo + ((int64_t)i - token * a.heads) * a.dim;
    for (int32_t d = lane * 8; d < a.dim; d += kWave * 8) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
        for (uint64_t rest = there; rest; rest &= rest - 1) {
            const int p = __builtin_ctzll(rest);
            const float by = read_lane(weight, p);
            Raw8<float> x;
            load_raw8(sums + (int64_t)p * a.dim + d, x);
            float z[8];
            widen8(x, z);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(z[e], by, y[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= inverse;
        store8(out + d, y);
    }
}

template <class T, int DP, bool FULL, bool BYPAGE>
static void launch_pieces(as_ctx *ctx, const AttendArgs &a, const AttendPieces &p, dim3 grid)
{
    const bool ragged = p.piece[0].mode == kAttendRagged;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, ctx->stream, a, p); };
    if (p.piece[0].mode == kAttendOwn) return launch(attend_own_kernel<T, DP, FULL, BYPAGE>);
    if constexpr (sizeof(T) == 2) {
        if (p.piece[0].queries == 128) {
            if (ragged) return launch(attend_tiles_kernel<DP, FULL, BYPAGE, kAttendRagged>);
            return launch(attend_tiles_kernel<DP, FULL, BYPAGE, kAttendShared>);
        }
    }
    if (ragged) return launch(attend_rows_kernel<T, DP, FULL, BYPAGE, kAttendRagged>);
    launch(attend_rows_kernel<T, DP, FULL, BYPAGE, kAttendShared>);
}
template <class T, int DP>
static void launch_pieces(as_ctx *ctx, const AttendArgs &a, const AttendPieces &p, dim3 grid)
{
    if (a.page_shift < 4) launch_pieces<T, DP, false, false>(ctx, a, p, grid);
    else if (a.dim != DP) launch_pieces<T, DP, false, true>(ctx, a, p, grid);
    else launch_pieces<T, DP, true, true>(ctx, a, p, grid);
}
template <class T>
static void launch_pieces(as_ctx *ctx, const AttendArgs &a, const AttendPieces &p, dim3 grid)
{
    if (a.dim <= 64) return launch_pieces<T, 64>(ctx, a, p, grid);
    if constexpr (sizeof(T) == 4) {
        // (fp32 products are bound by the matrix instructions: rows padded to less)
        if (a.dim <= 96) return launch_pieces<T, 96>(ctx, a, p, grid);
        if (a.dim > 128 && a.dim <= 192) return launch_pieces<T, 192>(ctx, a, p, grid);
    }
    if (a.dim <= 128) launch_pieces<T, 128>(ctx, a, p, grid);
    else launch_pieces<T, 256>(ctx, a, p, grid);
}

// Blocks of 256 threads that a launch takes: its threads are counted in 32 bits.
constexpr int64_t kMostBlocks = 0xffffffffLL / 256;

// Parts that the keys of each query are split into: two blocks a compute unit, if each still has `least` keys.  Joining costs all
// queries a pass over their parts, and prompts have many: they are split only where half of the units would have no block
// (8192 tokens in 416 blocks: 16 us whole, 37 in two parts; 1024 rows over shared prompts of 512 21 whole, 18 in two, 23 in four).
static int32_t parts_for(const as_ctx *ctx, int mode, int64_t blocks, int64_t room, int64_t least)
{
    int64_t n = mode == kAttendRagged ? ctx->num_cus / blocks : (2 * (int64_t)ctx->num_cus + blocks - 1) / blocks;
    const int64_t most = (room + least - 1) / least;
    n = n < most ? n : most;
    return (int32_t)(n < 1 ? 1 : n > kAttendMostParts ? kAttendMostParts : n);
}

static AttendPieces pieces_of(const as_ctx *ctx, const AttendArgs &a, int32_t *parts, bool *fit)
{
    AttendPieces p{};
    *parts = 0;
    // (a sequence's or a prompt's queries in 32 bits, and the blocks as a launch takes them)
    bool fits = a.tokens * a.group <= 0x7fffffffLL - 128 && a.per * (int64_t)a.group <= 0x7fffffffLL - 128;
    auto add = [&](int mode, int queries, int64_t groups, int32_t tiles, int64_t room) {
        AttendPiece &x = p.piece[p.count++];
        x.mode = mode;
        x.queries = queries;
        x.tiles = tiles;
        x.least = queries == 16 ? 8 : 4;
        x.part0 = *parts;
        x.parts = parts_for(ctx, mode, groups * tiles, room, 256);
        *parts += x.parts;
        fits = fits && groups * tiles <= 0x7fffffffLL;
        x.groups = (uint32_t)groups;
        x.items = x.blocks = (uint32_t)(groups * tiles);
        // Many short rows: one a wave, which spares them the joining of four.  us in blocks / in waves, 4 heads of 128, bf16: 512 of them
        // of up to 256 tokens 13.5 / 14.4; 1024 of up to 32, 128, 256, 512 9.3 / 5.9, 17.4 / 12.3, 24 / 20, 36 / 34; 2048 19 / 8.8, 30 / 20,
        // 41 / 36, 78 / 78; 8192 69 / 32, 121 / 88, 175 / 160, 291 / 297; fp32 1024 13 / 7.9, 26 / 20, 40 / 35, 78 / 77.
        x.alone = mode == kAttendOwn && x.parts == 1 && room <= 256 && groups * tiles >= 4 * (int64_t)ctx->num_cus;
        if (x.alone) x.blocks = (x.items + 3) / 4;
        fits = fits && (int64_t)x.blocks * x.parts <= kMostBlocks;
    };
    // Queries that share a key head, 16 or 128 a block (bf16): 128 take more time to start and less a query.  They pay where the 16s
    // are more blocks than the GPU takes at once, or read the keys too often: us for 16 / 128, dim 128, prompts of 1024 that rows of 32
    // queries share 2 of them 11.7 / 14.8, 16 of them 22.0 / 22.1, of 64 queries 36 / 24; of 8192 and 64 queries 131 / 69, 16 queries
    // 50 / 52; of 128 and 64 20 / 17; chunks of 16 queries behind 2000 tokens 4 of them 14 / 17, 64 of them 75 / 53; whole prompts of
    // 16, 32, 64, 256 queries, 64 of them, 7.3 / 8.3, 11.5 / 8.8, 16 / 9.6, 52 / 19.
    // (reads: blocks of 16 queries times the keys that each may have)
    auto by_128 = [&](int64_t blocks, int64_t most_blocks, double reads, int most_log) {
        if (a.dtype != AS_BF16 || ctx->attend_shape == 1) return false;
        return ctx->attend_shape == 2 || blocks > most_blocks || reads * a.dim >= (double)(1 << most_log);
    };
    if (a.offsets) {
        const int64_t all = a.tokens * a.group;
        const bool many = (all >= 16 * a.rows || ctx->attend_shape == 2) &&
                          by_128((all / 16 + a.rows) * a.kv_heads, 2 * (int64_t)ctx->num_cus, (double)all / 16 * a.kv_heads * a.room, 25);
        const int queries = many ? 128 : 16;
        add(kAttendRagged, queries, (all / queries + a.rows) * a.kv_heads, 1, a.room);
    } else {
        if (a.prompt_table) {
            const int64_t all = a.per * (int64_t)a.group, groups = (a.rows + a.per - 1) / a.per * a.kv_heads;
            const bool many = (all > 16 || ctx->attend_shape == 2) && by_128(groups * ((all + 15) / 16), (int64_t)ctx->num_cus - 1, (double)groups * ((all + 15) / 16) * a.prompt_room, 24);
            const int queries = many ? 128 : 16;
            add(kAttendShared, queries, groups, (int32_t)((all + queries - 1) / queries), a.prompt_room);
        }
        if (a.table) add(kAttendOwn, 16, a.rows * a.kv_heads, (a.group + 15) / 16, a.room);
    }
    p.every = 1;
    if (p.count == 2) {
        const int64_t first = (int64_t)p.piece[0].blocks * p.piece[0].parts, second = (int64_t)p.piece[1].blocks * p.piece[1].parts;
        p.every = (uint32_t)(1 + second / (2 * first)) | 1;        // (odd: blocks go round eight XCDs, and so then do every so many of them)
        fits = fits && first + second <= kMostBlocks;
    }
    // (and the queries' heads, where they are joined, four a block)
    *fit = fits && (*parts < 2 || a.tokens * a.heads <= 4 * kMostBlocks);
    return p;
}

size_t attend_workspace(const as_ctx *ctx, const AttendArgs &a)
{
    int32_t parts;
    bool fit;
    (void)pieces_of(ctx, a, &parts, &fit);
    return parts < 2 || !fit ? 0 : (size_t)a.tokens * a.heads * parts * (sizeof(float2) + (size_t)a.dim * sizeof(float));
}

as_status launch_attend(as_ctx *ctx, AttendArgs a)
{
    bool fit;
    const AttendPieces p = pieces_of(ctx, a, &a.parts, &fit);
    if (!fit) return fail(ctx, AS_ERR_UNSUPPORTED, "more queries than one launch takes");
    a.group_inverse = ((1u << 24) + a.group - 1) / a.group;
    a.sums = (float *)ctx->attend_parts.ptr;
    a.stats = (float2 *)(a.sums + (size_t)a.tokens * a.heads * a.parts * a.dim);
    int64_t blocks = 0;
    for (int i = 0; i < p.count; ++i) blocks += (int64_t)p.piece[i].blocks * p.piece[i].parts;
    if (a.dtype == AS_BF16) launch_pieces<uint16_t>(ctx, a, p, dim3((unsigned)blocks));
    else launch_pieces<float>(ctx, a, p, dim3((unsigned)blocks));
    AS_HIP_TRY(ctx, hipGetLastError());
    if (a.parts > 1) {
        const dim3 grid((unsigned)((a.tokens * a.heads + 3) / 4));
        if (a.dtype == AS_BF16) hipLaunchKernelGGL(attend_join_kernel<uint16_t>, grid, dim3(256), 0, ctx->stream, a);
        else hipLaunchKernelGGL(attend_join_kernel<float>, grid, dim3(256), 0, ctx->stream, a);
        AS_HIP_TRY(ctx, hipGetLastError());
    }
    return AS_OK;
}

// ---------------------------------------------------------------- new tokens

// Keys and values of new tokens into their sequences' pages, 16 bytes a thread and step: a token's heads lie one behind the other in
// the rows that a product leaves, and a page apart in the cache.  Token i of sequence s's n new ones goes to position
// lens[s] - n + i; what is outside the table or names no page is left out.  Bound by the memory (49000 tokens of 8 heads of 128, bf16:
// 89 us, 4.6 TB/s in and out), for a token a row by three loads after each other (1024 rows 3.8 us).  A token a block of a row each
// (eight: 6.8 us), eight of a prompt (one: 108).
__global__ __launch_bounds__(256) void cache_add_kernel(AttendArgs a, const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t tokens_each,
                                                        int32_t esz)
{
    const int32_t per_head = a.dim * esz / 16, pieces = 2 * a.kv_heads * per_head;
    int64_t s = 0, from = 0, to = 0, first;
    if (a.offsets) {
        const Found f = find_sequence<1>(a, blockIdx.x, 1, tokens_each);
        s = f.s;
        from = f.from;
        to = f.to;
        first = from + ((int64_t)blockIdx.x - s - from / tokens_each) * tokens_each;
        if (first < from || first >= to || (a.finished && a.finished[s])) return;
    } else {
        first = (int64_t)blockIdx.x * tokens_each;
        to = a.tokens;
    }
    const int32_t here = (int32_t)(to - first < tokens_each ? to - first : tokens_each);
    for (int32_t i = threadIdx.x; i < here * pieces; i += 256) {
        const int32_t t = i / pieces, x = i - t * pieces;
        const int64_t token = first + t, seq = a.offsets ? s : token;
        if (!a.offsets && a.finished && a.finished[seq]) continue;
        const int64_t pos = (int64_t)a.lens[seq] - (a.offsets ? to - token : 1);
        if (pos < 0 || pos >= a.room) continue;
        const int32_t page = a.table[seq * a.table_ld + (pos >> a.page_shift)];
        if (page < 0 || page >= a.pages) continue;
        const bool value = x >= pieces / 2;
        const int32_t y = value ? x - pieces / 2 : x, head = y / per_head, at = (y - head * per_head) * 16;
        const char *const source = (const char *)(value ? v : k) + token * (value ? ldv : ldk) * esz + (int64_t)y * 16;
        char *const target = (char *)const_cast<void *>(value ? a.v : a.k) + (uint64_t)(uint32_t)page * a.page_bytes +
                             (((int64_t)head << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * (int64_t)(a.dim * esz) + at;
        const u32x4_any in = *reinterpret_cast<const u32x4_any *>(source);
        *reinterpret_cast<u32x4 *>(target) = u32x4{in[0], in[1], in[2], in[3]};
    }
}

as_status launch_cache_add(as_ctx *ctx, const AttendArgs &a, const void *k, int64_t ldk, const void *v, int64_t ldv)
{
    const int32_t esz = a.dtype == AS_BF16 ? 2 : 4, pieces = 2 * a.kv_heads * (a.dim * esz / 16);
    int32_t each = (a.offsets ? 2048 : 256) / pieces;
    each = each < 1 ? 1 : each > 64 ? 64 : each;
    const int64_t blocks = a.offsets ? a.tokens / each + a.rows : (a.tokens + each - 1) / each;
    if (blocks > kMostBlocks) return fail(ctx, AS_ERR_UNSUPPORTED, "more tokens than one launch takes");
    hipLaunchKernelGGL(cache_add_kernel, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, a, k, ldk, v, ldv, each, esz);
    AS_HIP_TRY(ctx, hipGetLastError());
    return AS_OK;
}

}  // namespace as
