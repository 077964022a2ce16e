// Attention of new tokens over a paged cache of keys and values: causal, with an optional sliding window whose first tokens stay
// visible, over private pages and a prefix that all sequences share.
//
// For a row with query q: s_j = scale (q . k_j), out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) with the running maximum m: one
// pass over the keys and values, in which a larger maximum scales what has been added up so far.
#include "dc_device.h"
#include "dc_pages.h"

#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <type_traits>

using namespace dcpages;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int32_t kNoPosition = -0x40000000; // of a row that is not there: it sees nothing

// One part of the keys that a launch works through, the common prefix or the sequences' own pages, cut into n_splits runs of
// `chunk` tiles (the last one takes what is left).
struct Part {
    uint32_t blocks, n_splits, chunk, first_slot;
};

struct AttentionArgs {
    Batch batch;
    const void *k_pages, *v_pages, *q;
    void *out;
    float *lse;
    float *partial;    // [row][head][slot][head_dim]: sums of weight times value of one split, relative to its maximum
    f32x2 *partial_ml; // [row][head][slot]: that maximum (of scores in powers of two) and the sum of the weights
    uint64_t q_row, q_head, out_row, out_head;
    uint32_t n_heads, n_kv_heads, group, window, sinks, max_new, n_slots;
    float scale;       // above 0; with `negate` of queries that are taken with the other sign
    bool negate;
    bool whole;        // the prefix is read with the sequences' own pages, not as a part of its own
    Part prefix, own;
};

// kLiftFew, kLiftMany: by how many powers of two a row's reference lies below the largest score that it was taken from.  bf16 reaches as far
// down as fp32; f16 loses bits below 2^-14 and everything below 2^-25, which over a long context adds up to more than its unit (131071 keys:
// 0.4 %).  Its largest value is 2^16: in the kernel for few rows the largest weight is 2^15; in the one for many, whose reference lags
// behind the largest score, 2^7 to 2^15.  The sums are fp32 and have room for both.
template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    __device__ static __forceinline__ f32x4 m16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    __device__ static __forceinline__ f32x16 m32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static constexpr uint32_t kExponent = 0x7F80u;
    static constexpr float kLiftFew = 0.0f, kLiftMany = 0.0f;
};
template <> struct Mfma<_Float16> {
    __device__ static __forceinline__ f32x4 m16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    __device__ static __forceinline__ f32x16 m32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static constexpr uint32_t kExponent = 0x7C00u;
    static constexpr float kLiftFew = 15.0f, kLiftMany = 7.0f;
};

// Maximum and sum over the lanes with the same number modulo 16 (32).
__device__ __forceinline__ f32x2 swapped16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ f32x2 swapped32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float max_over_32(float v)
{
    const f32x2 r = swapped32(v);
    return fmaxf(r[0], r[1]);
}
__device__ __forceinline__ float max_over_16(float v)
{
    const f32x2 r = swapped16(v);
    return max_over_32(fmaxf(r[0], r[1]));
}
__device__ __forceinline__ float sum_over_16(float v)
{
    f32x2 r = swapped16(v);
    r = swapped32(r[0] + r[1]);
    return r[0] + r[1];
}

// Largest of the lanes' values.
__device__ __forceinline__ uint32_t largest_of_lanes(uint32_t v)
{
    v = max(v, dcdev::dpp_or_zero<0x111, 0xF>(v));
    v = max(v, dcdev::dpp_or_zero<0x112, 0xF>(v));
    v = max(v, dcdev::dpp_or_zero<0x114, 0xF>(v));
    v = max(v, dcdev::dpp_or_zero<0x118, 0xF>(v));
    v = max(v, dcdev::dpp_or_zero<0x142, 0xA>(v));
    v = max(v, dcdev::dpp_or_zero<0x143, 0xC>(v));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// Smallest and largest of the lanes' positions but kNoPosition; both are that if there is none.
__device__ __forceinline__ void range_of_positions(int32_t p_low, int32_t p_high, int32_t &low, int32_t &high)
{
    // positions are above kNoPosition (-2^30) by less than 2^31 + 2^30: counted from there, and down from 2^32 - 1, they have 0 for none
    high = (int32_t)(largest_of_lanes((uint32_t)p_high - (uint32_t)kNoPosition) + (uint32_t)kNoPosition);
    const uint32_t l = largest_of_lanes(p_low == kNoPosition ? 0u : ~((uint32_t)p_low - (uint32_t)kNoPosition));
    low = l ? (int32_t)(~l + (uint32_t)kNoPosition) : kNoPosition;
}

// 2^x; 0 for -infinity.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

// Of a block of 4 rows of 16 values of 16 bits that the 16 lanes name (a quarter of a row each), lane i gets column i.
__device__ __forceinline__ u32x2 lds_column4(uint32_t addr)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)addr));
}

// A value of V that is no number (an infinity, NaN) must reach only the rows that see its token, and a weight of 0 does not keep it from the
// others in a matrix product.  Where rows of one product differ in what they see, such values go into it as 0, and the rows that
// see their tokens get them by additions, from the cache once more.
template <typename T> __device__ __forceinline__ bool is_odd(uint32_t value) { return (value & Mfma<T>::kExponent) == Mfma<T>::kExponent; }
template <typename T> __device__ __forceinline__ u32x4 without_odd(u32x4 x)
{
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = (is_odd<T>(x[i]) ? 0u : x[i] & 0xFFFFu) | (is_odd<T>(x[i] >> 16) ? 0u : x[i] & 0xFFFF0000u);
    return x;
}
// Four neighbouring results of a row, with the values of a token that are no numbers added if the row sees it.
template <typename T> __device__ __forceinline__ f32x4 with_odd(f32x4 sum, const T *values, bool sees)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    const u32x2 x = *reinterpret_cast<const u32x2 *>(values);
    const f32x4 v = __builtin_convertvector(__builtin_bit_cast(T4, x), f32x4);
#pragma unroll
    for (int i = 0; i < 4; i++) sum[i] += (sees & is_odd<T>(x[i / 2] >> (16 * (i % 2)))) ? v[i] : 0.0f;
    return sum;
}
// The largest of 16-bit values without their signs says whether one of them is no number.
__device__ __forceinline__ u16x2 largest(u16x2 m, const u32x4 &x)
{
#pragma unroll
    for (int i = 0; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7FFF7FFFu));
    return m;
}

// The tokens of a part that a row at position p sees; positions count from the part's first token.
struct Seen {
    int32_t low, high, sinks;
    Seen() = default;
    __device__ __forceinline__ Seen(int32_t p, int32_t there, uint32_t window, int64_t sinks_left)
    {
        high = max(0, min(there, p + 1));
        low = window ? (int32_t)min((int64_t)high, max((int64_t)p - (int64_t)window + 1, (int64_t)0)) : 0;
        sinks = (int32_t)min((int64_t)high, max(sinks_left, (int64_t)0));
    }
    __device__ __forceinline__ bool token(int32_t j) const { return (j < high) & ((j >= low) | (j < sinks)); }
};

// The keys of one part that the rows of a workgroup see, as tiles of TILE tokens: the tiles with sinks, then those from the window's
// beginning on.  Positions here count from the part's first token.
template <int TILE> struct Tiles {
    int32_t low, high, sinks;   // tokens [0, sinks) and [low, high) are seen by some row
    int32_t low_tile, sink_tiles, count;
    // p_min, p_max: smallest and largest position of the rows, counted from the part's first token
    __device__ __forceinline__ Tiles(int32_t p_min, int32_t p_max, int32_t there, uint32_t window, int64_t sinks_left)
    {
        high = max(0, min(there, p_max + 1));
        const int64_t l = window ? (int64_t)p_min - (int64_t)window + 1 : 0;
        low = (int32_t)min((int64_t)high, max(l, (int64_t)0));
        sinks = (int32_t)min((int64_t)high, max(sinks_left, (int64_t)0));
        low_tile = low / TILE;
        sink_tiles = (sinks + TILE - 1) / TILE;
        if (low_tile <= sink_tiles) low_tile = 0, sink_tiles = 0;
        count = sink_tiles + max(0, (high + TILE - 1) / TILE - low_tile);
    }
    __device__ __forceinline__ int32_t first_token(int32_t tile) const { return (tile < sink_tiles ? tile : low_tile + tile - sink_tiles) * TILE; }
};

// Results of a row and head: v holds four sums of weight times value, relative to the maximum m, l the sum of the weights.
template <typename T> __device__ __forceinline__ void store_whole(const AttentionArgs &a, uint32_t row, uint32_t head, uint32_t at, f32x4 v, float m, float l)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    const float r = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    *reinterpret_cast<T4 *>(static_cast<T *>(a.out) + row * a.out_row + head * a.out_head + at) =
        __builtin_convertvector(l == 0.0f ? f32x4{} : v * r, T4);
    if (a.lse && at == 0) a.lse[(uint64_t)row * a.n_heads + head] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
// The same, or if it is one of several splits what they are joined from.
template <typename T, int D> __device__ __forceinline__ void store_result(const AttentionArgs &a, uint32_t row, uint32_t head, uint32_t slot,
                                                                          uint32_t at, f32x4 v, float m, float l)
{
    if (a.n_slots == 1) {
        store_whole<T>(a, row, head, at, v, m, l);
    } else {
        const uint64_t i = ((uint64_t)row * a.n_heads + head) * a.n_slots + slot;
        *reinterpret_cast<f32x4 *>(a.partial + i * D + at) = v;
        if (at == 0) a.partial_ml[i] = f32x2{m, l};
    }
}

// ---- few rows -------------------------------------------------------------------------------------------------------------
//
// At most 16 RT rows (new tokens times the query heads that share a key/value head) read the keys: memory bounds this kernel.  A
// wavefront takes tiles of 32 tokens.  Scores come as a matrix [token][row] = K Q^T from 16x16x32 products, whose first operand is
// K as it lies in memory: a lane holds 8 neighbouring values of a token.  In the result a lane holds 4 tokens of one row in each
// half of the tile, which is already the second operand of [head_dim][row] = V^T P^T if the product's 32 tokens are numbered that way; the
// first operand, 8 tokens of one value, comes out of the LDS through the transposing read.  So maxima, sums and the scaling of
// what has been added up stay inside a lane but for two exchanges a tile.  K and then V go through registers into the wavefront's
// own part of the LDS: no barrier in the loop.  The next tile's loads are under way during the rest of the tile's work.
// One token over 131071 tokens, 537 MB: 80.5 us (6.7 TB/s) and 4.5 for the join; 64 sequences of 512 to 8192 tokens, 1.2 GB: 205 us (5.85 TB/s, for
// sequences of unlike lengths end at unlike times; alike ones read 6.6); one token over 1999, 32 heads: 8 us and 3.
template <int D, int RT> struct FewLds {
    static constexpr int kPadded = D + 4; // floats of a row's sums
    union {
        uint8_t tokens[4][32 * 2 * D]; // of each wavefront: a tile's keys, then its values
        float sums[4][16][kPadded];
    };
    float m[4][16 * RT], l[4][16 * RT];
    int32_t p[16 * RT];
};

template <typename T, int D, int RT> __device__ __forceinline__ void few_rows(const AttentionArgs &a, FewLds<D, RT> &lds, bool common, uint32_t item)
{
    typedef typename Vec8<T>::type TV;
    constexpr int kTile = 32, KS = D / 32, DT = D / 16;
    constexpr int kRowBytes = 2 * D, kChunks = D / 8, kRowsALoad = 64 / kChunks, kLoads = kTile / kRowsALoad;

    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15u, g = lane >> 4;
    const Part &part = common ? a.prefix : a.own;
    const uint32_t kv = item % a.n_kv_heads;
    item /= a.n_kv_heads;
    const uint32_t seq = common ? 0 : item % a.batch.n_seqs, split = common ? item : item / a.batch.n_seqs;
    const int32_t *table = common ? a.batch.prefix_pages : a.batch.pages + (uint64_t)seq * a.batch.pages_stride;
    const uint32_t table_entries = common ? (a.batch.prefix_len + (1u << a.batch.page_shift) - 1) >> a.batch.page_shift : a.batch.pages_stride;
    // entries of a tile's two halves
    auto entries_at = [&](uint32_t j, int32_t (&entry)[2]) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t i = (j + 16 * h) >> a.batch.page_shift;
            entry[h] = i < table_entries ? table[i] : -1;
        }
    };
    // Without a window it is known at once where a wavefront's first tile is: its pages are asked for together with the sequence's length.
    int32_t first_entry[2] = {-1, -1};
    const uint64_t first_tile = (uint64_t)split * part.chunk + wave;
    if (!a.window && first_tile < 1u << 26) entries_at((uint32_t)first_tile * kTile, first_entry);

    // rows of this workgroup: row_first + i / group of head kv * group + i % group for i < n
    uint32_t row_first = 0, n;
    int32_t p_first = 0, there, base = 0, p_min, p_max;
    if (common) {
        n = a.batch.n_rows * a.group;
        there = (int32_t)a.batch.prefix_len;
        // positions of the rows, sequence by sequence
        if (threadIdx.x < 16 * RT) lds.p[threadIdx.x] = kNoPosition;
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < a.batch.n_seqs; b += 256) {
            const uint32_t first = a.batch.first_row(b), end = a.batch.rows_end(b);
            for (uint32_t r = first; r < end; r++) lds.p[r] = a.batch.length(b) - (int32_t)(end - r);
        }
        __syncthreads();
        const int32_t p = lane < min(a.batch.n_rows, 16u * RT) ? lds.p[lane] : kNoPosition;
        range_of_positions(p, p, p_min, p_max);
    } else {
        row_first = a.batch.first_row(seq);
        const uint32_t end = a.batch.rows_end(seq);
        const int32_t len = a.batch.length(seq);
        if (end <= row_first) return;
        const uint32_t rows = min(end - row_first, a.max_new);
        n = rows * a.group;
        base = (int32_t)a.batch.prefix_len;
        there = min(max(len - base, 0), (int32_t)(a.batch.pages_stride << a.batch.page_shift));
        p_first = len - (int32_t)(end - row_first);
        p_min = p_first - base, p_max = p_first + (int32_t)rows - 1 - base;
    }
    const Tiles<kTile> tiles(p_min, p_max, there, a.window, (int64_t)a.sinks - base);
    const int32_t t_begin = (int32_t)min((uint64_t)split * part.chunk, (uint64_t)tiles.count);
    const int32_t t_end = split + 1 == part.n_splits ? tiles.count : (int32_t)min((uint64_t)t_begin + part.chunk, (uint64_t)tiles.count);

    // queries, and what the lane's rows see
    TV q[RT][KS];
    Seen seen[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const uint32_t r = rt * 16 + c;
        const bool is = r < n;
        const uint32_t i = r / a.group, head = kv * a.group + r % a.group;
        seen[rt] = Seen(!is ? kNoPosition : common ? lds.p[i] : p_first + (int32_t)i - base, there, a.window, (int64_t)a.sinks - base);
        const T *src = static_cast<const T *>(a.q) + (uint64_t)(row_first + i) * a.q_row + head * a.q_head + 8 * g;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            u32x4 x = {};
            if (is) x = *reinterpret_cast<const u32x4 *>(src + 32 * s);
            if (a.negate) x ^= 0x80008000u;
            q[rt][s] = __builtin_bit_cast(TV, x);
        }
    }

    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        m[rt] = -INFINITY, l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) o[rt][dt] = f32x4{};
    }

    const uint64_t page_stride = (uint64_t)a.n_kv_heads << a.batch.page_shift;
    const uint64_t head_at = (uint64_t)kv << a.batch.page_shift;
    const uint32_t place_mask = (1u << a.batch.page_shift) - 1u;
    // page of each half of a tile, -1 where there is none
    auto pages_from = [&](const int32_t (&entry)[2], int32_t (&page)[2]) {
#pragma unroll
        for (int h = 0; h < 2; h++) page[h] = __builtin_amdgcn_readfirstlane((uint32_t)entry[h] < a.batch.n_pages ? entry[h] : -1);
    };
    auto pages_of = [&](int32_t tile, int32_t (&page)[2]) {
        int32_t entry[2];
        entries_at((uint32_t)tiles.first_token(tile), entry);
        pages_from(entry, page);
    };
    // first value of a half's tokens; where there is no page, of page 0, whose tokens are then taken for hidden
    auto half_at = [&](int32_t j, int32_t page) {
        return (page_stride * (uint32_t)max(page, 0) + head_at + ((uint32_t)j & place_mask)) * D;
    };
    u32x4 k[kLoads], v[kLoads];
    // A tile's keys or values in the order of memory, whole tokens side by side; nothing else will ask for them.
    auto load = [&](u32x4 (&to)[kLoads], const void *pages, int32_t j, const int32_t (&page)[2]) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const T *src = static_cast<const T *>(pages) + half_at(j + 16 * h, page[h]) + lane * 8;
#pragma unroll
            for (int i = 0; i < kLoads / 2; i++) to[h * (kLoads / 2) + i] = dcdev::load16_stream(src + i * 512);
        }
    };
    // Tokens lie in the LDS with their 16-byte chunks exchanged so that 8 tokens' same chunks, and pairs of chunks, are on different banks.
    auto swizzle = [](uint32_t row) { return D == 64 ? ((row >> 1) & 3u) << 1 : (row & 7u) << 1; };
    const uint32_t my_lds = dcdev::lds_address(lds.tokens[wave]);
    auto put = [&](const u32x4 (&from)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t row = i * kRowsALoad + lane / kChunks, chunk = lane % kChunks;
            *(lds_u32x4 *)(uintptr_t)(my_lds + row * kRowBytes + ((chunk ^ swizzle(row)) << 4)) = from[i];
        }
        __builtin_amdgcn_wave_barrier();
    };

    int32_t page[2], next_page[2];
    int32_t t = t_begin + (int32_t)wave;
    if (t < t_end) {
        if (a.window) pages_of(t, page);
        else pages_from(first_entry, page);
        const int32_t j = tiles.first_token(t);
        load(k, a.k_pages, j, page);
        load(v, a.v_pages, j, page);
        pages_of(min(t + 4, t_end - 1), next_page);
    }
    for (; t < t_end; t += 4) {
        const int32_t j = tiles.first_token(t);
        const bool more = t + 4 < t_end;
        const int32_t next_j = tiles.first_token(min(t + 4, t_end - 1));

        put(k);
        if (more) load(k, a.k_pages, next_j, next_page);
        f32x4 s[RT][2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
#pragma unroll
            for (int rt = 0; rt < RT; rt++) s[rt][h] = f32x4{};
#pragma unroll
            for (int i = 0; i < KS; i++) {
                const uint32_t row = 16 * h + c, chunk = 4 * i + g;
                const TV x = __builtin_bit_cast(TV, *(const lds_u32x4 *)(uintptr_t)(my_lds + row * kRowBytes + ((chunk ^ swizzle(row)) << 4)));
#pragma unroll
                for (int rt = 0; rt < RT; rt++) s[rt][h] = Mfma<T>::m16(x, q[rt][i], s[rt][h]);
            }
        }
        __builtin_amdgcn_wave_barrier();

        // tokens that not all rows see; those that none sees lie in the LDS as zeros
        const bool edge = page[0] < 0 || page[1] < 0 || j + kTile > p_min + 1 || j + kTile > tiles.high || (j < tiles.low && j + kTile > tiles.sinks) ||
                          (a.window && j + kTile > tiles.sinks && (int64_t)j <= (int64_t)p_max - a.window);
        if (edge) {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const int32_t jj = j + i * kRowsALoad + (int32_t)(lane / kChunks);
                const bool some = (page[i >= kLoads / 2] >= 0) & (jj < tiles.high) & ((jj >= tiles.low) | (jj < tiles.sinks));
                v[i] = some ? v[i] : u32x4{};
            }
        }
        bool odd = false; // a value that is no number, which some rows see and others do not
        if (edge && p_min != p_max) {
            u16x2 most = {};
#pragma unroll
            for (int i = 0; i < kLoads; i++) most = largest(most, v[i]);
            odd = __any((most[0] >= Mfma<T>::kExponent) | (most[1] >= Mfma<T>::kExponent));
            if (odd) {
#pragma unroll
                for (int i = 0; i < kLoads; i++) v[i] = without_odd<T>(v[i]);
            }
        }
        put(v);
        if (more) load(v, a.v_pages, next_j, next_page);

        TV w[RT];
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            if (edge) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool sees = seen[rt].token(j + 16 * h + 4 * (int32_t)g + i) & (page[h] >= 0);
                        s[rt][h][i] = sees ? s[rt][h][i] : -INFINITY;
                    }
            }
            float top = fmaxf(fmaxf(fmaxf(s[rt][0][0], s[rt][0][1]), fmaxf(s[rt][0][2], s[rt][0][3])),
                              fmaxf(fmaxf(s[rt][1][0], s[rt][1][1]), fmaxf(s[rt][1][2], s[rt][1][3])));
            top = fmaxf(m[rt], max_over_16(top));
            const float ref = top == -INFINITY ? 0.0f : top;
            const float fade = exp2_of((m[rt] - ref) * a.scale);
            m[rt] = top;
            typedef float f32x8 __attribute__((ext_vector_type(8)));
            f32x8 e;
#pragma unroll
            for (int i = 0; i < 8; i++) e[i] = exp2_of(__builtin_fmaf(s[rt][i / 4][i % 4] - ref, a.scale, Mfma<T>::kLiftFew));
            l[rt] = l[rt] * fade + (((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
            w[rt] = __builtin_convertvector(e, TV);
#pragma unroll
            for (int dt = 0; dt < DT; dt++) o[rt][dt] *= fade;
        }
        const uint32_t i4 = c >> 2, half8 = (c & 1u) << 3;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) {
            const uint32_t row = 4 * g + i4, chunk = 2 * dt + ((c & 3u) >> 1);
            const uint32_t at = my_lds + row * kRowBytes + ((chunk ^ swizzle(row)) << 4) + half8;
            const u32x2 lo = lds_column4(at), hi = lds_column4(at + 16 * kRowBytes);
            const u32x4 x = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int rt = 0; rt < RT; rt++) o[rt][dt] = Mfma<T>::m16(__builtin_bit_cast(TV, x), w[rt], o[rt][dt]);
        }
        if (odd) {
#pragma unroll 1
            for (int i = 0; i < kTile; i++) {
                if (page[i / 16] < 0) continue;
                const T *src = static_cast<const T *>(a.v_pages) + half_at(j + i, page[i / 16]) + 4 * g;
#pragma unroll
                for (int rt = 0; rt < RT; rt++)
#pragma unroll
                    for (int dt = 0; dt < DT; dt++) o[rt][dt] = with_odd<T>(o[rt][dt], src + 16 * dt, seen[rt].token(j + i));
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; h++) page[h] = next_page[h];
        if (more) pages_of(min(t + 8, t_end - 1), next_page);
    }

    // the wavefronts' sums, brought to one maximum and added up in their order
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        l[rt] = sum_over_16(l[rt]);
        m[rt] = m[rt] * a.scale - Mfma<T>::kLiftFew; // what the weights are relative to
        if (l[rt] != l[rt] && m[rt] == -INFINITY) m[rt] = 0.0f; // saw scores, none of them a number
        if (g == 0) lds.m[wave][rt * 16 + c] = m[rt], lds.l[wave][rt * 16 + c] = l[rt];
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const uint32_t r = rt * 16 + c;
        const float top = fmaxf(fmaxf(lds.m[0][r], lds.m[1][r]), fmaxf(lds.m[2][r], lds.m[3][r]));
        const float f = m[rt] == -INFINITY ? 0.0f : exp2_of(m[rt] - top);
        if (rt) __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
            *reinterpret_cast<f32x4 *>(&lds.sums[wave][c][16 * dt + 4 * g]) = m[rt] == -INFINITY ? f32x4{} : o[rt][dt] * f;
        __syncthreads();
        constexpr uint32_t kQuads = D / 4;
        for (uint32_t i = threadIdx.x; i < 16 * kQuads; i += 256) {
            const uint32_t col = i / kQuads, at = i % kQuads * 4, rr = rt * 16 + col;
            if (rr >= n) continue;
            const float big = fmaxf(fmaxf(lds.m[0][rr], lds.m[1][rr]), fmaxf(lds.m[2][rr], lds.m[3][rr]));
            f32x4 sum = {};
            float total = 0.0f;
#pragma unroll
            for (int w4 = 0; w4 < 4; w4++) {
                sum += *reinterpret_cast<const f32x4 *>(&lds.sums[w4][col][at]);
                if (lds.m[w4][rr] != -INFINITY) total += lds.l[w4][rr] * exp2_of(lds.m[w4][rr] - big);
            }
            store_result<T, D>(a, row_first + rr / a.group, kv * a.group + rr % a.group, part.first_slot + split, at, sum, big, total);
        }
    }
}

template <typename T, int D, int RT> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void dc_attention_few_kernel(AttentionArgs a)
{
    __shared__ __align__(16) FewLds<D, RT> lds;
    const bool common = blockIdx.x < a.prefix.blocks;
    few_rows<T, D, RT>(a, lds, common, common ? blockIdx.x : blockIdx.x - a.prefix.blocks);
}


constexpr uint32_t kTileRows = 128; // of a workgroup of the kernel for many rows

// ---- many rows ------------------------------------------------------------------------------------------------------------
//
// A workgroup owns 128 rows of one key/value head (prompts, or the rows of many sequences behind a common prefix): the matrix
// units bound this kernel.  Keys and values go through the LDS in tiles that its four wavefronts share, double buffered with one barrier a
// tile; a wavefront owns 32 rows.  The products are those of the kernel for few rows in the 32x32x16 shape: scores as [token][row]
// = K Q^T, of which a lane holds 16 of 32 tokens of one row, results as [head_dim][row] = V^T P^T; maxima and sums stay in a lane but for one
// exchange between the halves.  A prompt of 8192 tokens, 32 heads of 128: 580 to 600 us for as long as it runs (915 to 945 TFLOP/s; a large library
// product reaches 1250; the first 40 launches after an idle time up to 770 us, while the clock settles), the matrix units busy 44 % and the
// vector units 42 % of the cycles at a clock that falls to 2.0 GHz.  Tiles of 64 tokens are 8 to 20 % faster than of 32, for which
// alone heads of 256 have registers (590 to 600 TFLOP/s).
template <int D> struct TileLds {
    static constexpr int kTile = D == 256 ? 32 : 64; // tokens
    uint8_t k[2][kTile * 2 * D], v[2][kTile * 2 * D];
    int32_t p[kTileRows];
    uint32_t odd[2][4];
};

template <typename T, int D> __device__ __forceinline__ void many_rows(const AttentionArgs &a, TileLds<D> &lds, bool common, uint32_t block)
{
    typedef typename Vec8<T>::type TV;
    constexpr int kTile = TileLds<D>::kTile, KS = D / 16, DT = D / 32, HT = kTile / 32; // HT: 32-token products of a tile
    constexpr uint32_t kRows = kTileRows, kRowBytes = 2 * D, kChunks = D / 8, kRowsALoad = 64 / kChunks;
    constexpr int kTokens = kTile / 4, kLoads = kTokens / (int)kRowsALoad; // tokens that a wavefront brings, in so many loads
    constexpr uint32_t kBuffer = kTile * kRowBytes;

    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31u, half = lane >> 5;
    const Part &part = common ? a.prefix : a.own;
    uint32_t item = part.blocks - 1 - block; // the last rows, which see most, first
    const uint32_t kv = a.n_kv_heads - 1 - item % a.n_kv_heads;
    item /= a.n_kv_heads;
    const uint32_t split = part.n_splits - 1 - item % part.n_splits;
    uint32_t tile = item / part.n_splits;

    // rows of this workgroup: i_first <= i < n of the sequence's (the batch's) rows, row_first + i / group of head kv * group + i % group
    uint32_t row_first = 0, n = 0, seq = 0;
    int32_t there = (int32_t)a.batch.prefix_len; // positions below it are, or may be, in the cache
    int32_t p_first = 0;                         // of the sequence's first row
    if (common) {
        n = a.batch.n_rows * a.group;
    } else {
        // a lane to a sequence: how many workgroups it has, and so whose this one is
        bool found = false;
        uint32_t end = 0;
        int32_t len = 0;
        if (a.batch.row_start) {
            for (uint32_t b = 0; b < a.batch.n_seqs && !found; b += 64) {
                const uint32_t s = min(b + lane, a.batch.n_seqs - 1), first_s = a.batch.first_row(s), end_s = a.batch.rows_end(s);
                const int32_t len_s = a.batch.length(s);
                const uint32_t tiles = b + lane < a.batch.n_seqs && end_s > first_s ? (min(end_s - first_s, a.max_new) * a.group + kRows - 1) / kRows : 0;
                const uint32_t upto = dcdev::lanes_prefix_sum<false>(tiles);
                const uint64_t beyond = __ballot(upto > tile);
                if (beyond) {
                    const int l = __builtin_ctzll(beyond);
                    seq = b + (uint32_t)l;
                    tile -= (uint32_t)__builtin_amdgcn_readlane((int)(upto - tiles), l);
                    row_first = (uint32_t)__builtin_amdgcn_readlane((int)first_s, l);
                    end = (uint32_t)__builtin_amdgcn_readlane((int)end_s, l);
                    len = __builtin_amdgcn_readlane(len_s, l);
                    found = true;
                } else {
                    tile -= (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
                }
            }
        } else {
            const uint32_t tiles = (a.group + kRows - 1) / kRows;
            seq = tile / tiles, tile %= tiles;
            found = seq < a.batch.n_seqs;
            if (found) row_first = seq, end = seq + 1, len = a.batch.length(seq);
        }
        if (!found) return;
        seq = __builtin_amdgcn_readfirstlane(seq), tile = __builtin_amdgcn_readfirstlane(tile);
        n = min(end - row_first, a.max_new) * a.group;
        p_first = len - (int32_t)(end - row_first);
        there = max(there, min(len, a.batch.capacity()));
    }
    const uint32_t i_first = tile * kRows;

    // positions of the rows: of a sequence they follow from one another; of the batch they are gathered, sequence by sequence
    int32_t p_min, p_max, wave_p_min, wave_p_max, my_p;
    const uint32_t my_row = i_first + wave * 32 + c;
    if (common) {
        for (uint32_t i = threadIdx.x; i < kRows; i += 256) lds.p[i] = kNoPosition;
        __syncthreads();
        const uint32_t r_low = i_first / a.group, r_high = min((i_first + kRows - 1) / a.group + 1, a.batch.n_rows);
        for (uint32_t b = threadIdx.x; b < a.batch.n_seqs; b += 256) {
            const uint32_t first = a.batch.first_row(b), end = a.batch.rows_end(b);
            const int32_t len = first < end ? a.batch.length(b) : 0;
            for (uint32_t r = max(first, r_low); r < min(end, r_high); r++)
                for (uint32_t i = max(r * a.group, i_first); i < min((r + 1) * a.group, i_first + kRows); i++) lds.p[i - i_first] = len - (int32_t)(end - r);
        }
        __syncthreads();
        const int32_t p0 = lds.p[lane], p1 = lds.p[lane + 64];
        range_of_positions(p0 == kNoPosition ? p1 : p1 == kNoPosition ? p0 : min(p0, p1), max(p0, p1), p_min, p_max);
        const int32_t p = lds.p[wave * 32 + c];
        range_of_positions(p, p, wave_p_min, wave_p_max);
        my_p = lds.p[wave * 32 + c];
    } else {
        auto position = [&](uint32_t i) { return i < n ? p_first + (int32_t)(i / a.group) : kNoPosition; };
        const uint32_t wave_first = i_first + wave * 32;
        p_min = position(i_first), p_max = position(min(i_first + kRows, n) - 1);
        wave_p_min = position(wave_first), wave_p_max = wave_first < n ? position(min(wave_first + 32, n) - 1) : kNoPosition;
        my_p = position(my_row);
    }
    // The tiles of the common prefix, if it is this launch's to read here, and behind them those of the sequence's own pages, whose first token
    // is at `base`.  Positions count from the sequence's first token, but in the two tables of pages.
    const int32_t base = (int32_t)a.batch.prefix_len;
    auto beyond = [&](int32_t p) { return (int32_t)max((int64_t)p - base, (int64_t)-1); };
    const Tiles<kTile> prefix_tiles(p_min, p_max, common || a.whole ? base : 0, a.window, a.sinks);
    const Tiles<kTile> own_tiles(beyond(p_min), beyond(p_max), common ? 0 : there - base, a.window, (int64_t)a.sinks - base);
    const int32_t count = prefix_tiles.count + own_tiles.count;
    const int32_t t_begin = (int32_t)min((uint64_t)split * part.chunk, (uint64_t)count);
    const int32_t t_end = split + 1 == part.n_splits ? count : (int32_t)min((uint64_t)t_begin + part.chunk, (uint64_t)count);
    auto first_token = [&](int32_t t) { return t < prefix_tiles.count ? prefix_tiles.first_token(t) : base + own_tiles.first_token(t - prefix_tiles.count); };
    const Seen all_first(p_min, there, a.window, a.sinks), all_last(p_max, there, a.window, a.sinks); // of the workgroup's rows
    const Seen first_sees(wave_p_min, there, a.window, a.sinks), last_sees(wave_p_max, there, a.window, a.sinks); // of the wavefront's

    const uint32_t my_head = kv * a.group + my_row % a.group;
    const uint64_t my_packed = row_first + my_row / a.group;
    const Seen seen(my_p, there, a.window, a.sinks);
    TV q[KS];
    f32x16 o[DT];
    f32x16 below = f32x16{}; // the reference with the other sign, in every value
    bool any = false;        // a score has been seen
    float l = 0.0f;
    const T *q_src = static_cast<const T *>(a.q) + my_packed * a.q_row + my_head * a.q_head + 8 * half;
#pragma unroll
    for (int i = 0; i < KS; i++) {
        u32x4 x = {};
        if (my_row < n) x = *reinterpret_cast<const u32x4 *>(q_src + 16 * i);
        if (a.negate) x ^= 0x80008000u;
        q[i] = __builtin_bit_cast(TV, x);
    }
#pragma unroll
    for (int dt = 0; dt < DT; dt++) o[dt] = f32x16{};

    const int32_t *prefix_table = a.batch.prefix_pages, *own_table = a.batch.pages + (uint64_t)seq * a.batch.pages_stride;
    const uint64_t page_stride = (uint64_t)a.n_kv_heads << a.batch.page_shift;
    const uint64_t head_at = (uint64_t)kv << a.batch.page_shift;
    const uint32_t place_mask = (1u << a.batch.page_shift) - 1u;
    // What there is to know of 16 tiles, 16 tiles ahead: lane l has, of tile i + l / 4 counted from t_begin, where the tokens that wavefront l mod 4
    // brings lie in the pools (in bytes; where there is no page, those of page 0, which are then taken for hidden), and the tile's
    // flags.  A tile's step takes its own with three reads of a lane.  (Scalar loads would do for the pages, but the LDS's data are waited
    // for by the same counter, all of it.)
    enum : uint32_t {
        kThere = 15,    // a bit for each wavefront's tokens: they are there
        kPrefix = 16,   // of the prefix's table
        kPartial = 32,  // not all rows of the workgroup see all of it
        kSome = 64,     // this wavefront's rows see some of it,
        kEdge = 128     // and not all of it
    };
    struct Known {
        uint32_t low, high, flags;
    };
    auto pages_from = [&](int32_t i) {
        const int32_t t = t_begin + i + (int32_t)(lane >> 2), j = first_token(t) + (int32_t)(lane & 3u) * kTokens;
        const bool in_prefix = t < prefix_tiles.count;
        int32_t e = -1;
        if (t < t_end && j < (in_prefix ? base : all_last.high)) e = in_prefix ? prefix_table[(uint32_t)j >> a.batch.page_shift] : own_table[(uint32_t)(j - base) >> a.batch.page_shift];
        return (uint32_t)e < a.batch.n_pages ? e : -1;
    };
    auto known_from = [&](int32_t i, int32_t page) {
        const int32_t t = t_begin + i + (int32_t)(lane >> 2), j = first_token(t);
        const bool in_prefix = t < prefix_tiles.count;
        const uint32_t place = (uint32_t)(j + (int32_t)(lane & 3u) * kTokens - (in_prefix ? 0 : base)) & place_mask;
        const uint64_t at = (page_stride * (uint32_t)max(page, 0) + head_at + place) * kRowBytes;
        const uint32_t there4 = (uint32_t)(__ballot(page >= 0) >> (lane & 60u)) & 15u;
        const bool whole = there4 == 15u && (!in_prefix || j + kTile <= base);
        const bool partial = !whole || j + kTile > all_first.high || j < all_last.low;
        const bool some = t < t_end && j < last_sees.high && (j + kTile > first_sees.low || j < last_sees.sinks);
        const bool edge = !whole || j + kTile > first_sees.high || (j < last_sees.low && j + kTile > first_sees.sinks);
        return Known{(uint32_t)at, (uint32_t)(at >> 32), there4 | (in_prefix ? kPrefix : 0u) | (partial ? kPartial : 0u) | (some ? kSome : 0u) | (edge ? kEdge : 0u)};
    };
    int32_t pages_ahead = pages_from(0);
    Known known = known_from(0, pages_ahead);
    pages_ahead = pages_from(16);
    auto flags_of = [&](int32_t i) { return (uint32_t)__builtin_amdgcn_readlane((int)known.flags, 4 * (i & 15)); };
    // tokens from here on are not of the tile's table
    auto end_of = [&](uint32_t flags) { return flags & kPrefix ? base : 0x7FFFFFFF; };
    u32x4 k_new[kLoads], v_new[kLoads];
    const uint32_t lane_at = lane * 16;
    auto bring = [&](int32_t i) {
        const int32_t l = 4 * (i & 15) + (int32_t)wave;
        const uint64_t at = (uint32_t)__builtin_amdgcn_readlane((int)known.low, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)known.high, l) << 32;
        const uint8_t *k_at = static_cast<const uint8_t *>(a.k_pages) + at, *v_at = static_cast<const uint8_t *>(a.v_pages) + at;
#pragma unroll
        for (int i = 0; i < kLoads; i++) k_new[i] = *reinterpret_cast<const u32x4 *>(k_at + lane_at + i * 1024);
#pragma unroll
        for (int i = 0; i < kLoads; i++) v_new[i] = *reinterpret_cast<const u32x4 *>(v_at + lane_at + i * 1024);
    };
    // The 16-byte chunks of a token lie exchanged in the LDS, so that 16 tokens' same chunks are on different banks, and the same four of 4 tokens'.
    auto swizzle = [](uint32_t token) {
        return D == 64 ? (token >> 1 & 1u) << 2 | (token >> 2 & 3u) : (token & 3u) << 2 | (token >> 2 & 3u);
    };
    const uint32_t lds_k = dcdev::lds_address(&lds) + offsetof(TileLds<D>, k), lds_v = dcdev::lds_address(&lds) + offsetof(TileLds<D>, v);
    // where a lane puts what it brings, and where it reads its part of the first operands
    uint32_t put_at[kLoads], k_at[KS], v_at[DT][2];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const uint32_t token = wave * kTokens + i * kRowsALoad + lane / kChunks, chunk = lane % kChunks;
        put_at[i] = token * kRowBytes + ((chunk ^ swizzle(token)) << 4);
    }
#pragma unroll
    for (int i = 0; i < KS; i++) k_at[i] = c * kRowBytes + (((2 * i + half) ^ swizzle(c)) << 4);
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t i16 = lane & 15u, token = 4 * half + (i16 >> 2) + 8 * h, chunk = 4 * dt + 2 * (lane >> 4 & 1u) + (i16 >> 1 & 1u);
            v_at[dt][h] = token * kRowBytes + ((chunk ^ swizzle(token)) << 4) + (i16 & 1u) * 8;
        }
    auto put_k = [&](uint32_t buffer) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) *(lds_u32x4 *)(uintptr_t)(lds_k + buffer * kBuffer + put_at[i]) = k_new[i];
    };
    // Of a partial tile a wavefront leaves in lds.odd whether one of the values of V that it brought is no number.
    auto put_v = [&](int32_t t, uint32_t flags, uint32_t buffer) {
        if (flags & kPartial) {
            const bool is_there = (flags >> wave & 1u) != 0;
            const int32_t j = first_token(t) + (int32_t)wave * kTokens;
            u16x2 most = {};
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const int32_t jj = j + i * (int32_t)kRowsALoad + (int32_t)(lane / kChunks);
                const bool some = is_there & (jj < min(end_of(flags), all_last.high)) & ((jj >= all_first.low) | (jj < all_last.sinks));
                v_new[i] = some ? v_new[i] : u32x4{};
                most = largest(most, v_new[i]);
            }
            const bool odd = __any((most[0] >= Mfma<T>::kExponent) | (most[1] >= Mfma<T>::kExponent));
            if (odd) {
#pragma unroll
                for (int i = 0; i < kLoads; i++) v_new[i] = without_odd<T>(v_new[i]);
            }
            if (lane == 0) lds.odd[buffer][wave] = odd;
        }
#pragma unroll
        for (int i = 0; i < kLoads; i++) *(lds_u32x4 *)(uintptr_t)(lds_v + buffer * kBuffer + put_at[i]) = v_new[i];
    };
    auto k_operand = [&](int i, uint32_t buffer) {
        return __builtin_bit_cast(TV, *(const lds_u32x4 *)(uintptr_t)(lds_k + buffer * kBuffer + 32 * (i / KS) * kRowBytes + k_at[i % KS]));
    };
    auto v_operand = [&](int i, uint32_t buffer) {
        const u32x2 lo = lds_column4(lds_v + buffer * kBuffer + 16 * (i / DT) * kRowBytes + v_at[i % DT][0]);
        const u32x2 hi = lds_column4(lds_v + buffer * kBuffer + 16 * (i / DT) * kRowBytes + v_at[i % DT][1]);
        return __builtin_bit_cast(TV, u32x4{lo[0], lo[1], hi[0], hi[1]});
    };

    // A step works on tile t, whose keys and values are in buffer B, while the next tile's go from registers into the other buffer and those
    // of the tile behind it are asked for.
    uint32_t flags = 0, flags_next = 0; // of tiles t and t + 1
    auto step = [&](auto B, int32_t t) {
        constexpr uint32_t buffer = decltype(B)::value;
        constexpr int kProducts = HT * KS, kGroups = 2 * HT, kAhead = 4;
        if (t + 1 < t_end) {
            put_k(buffer ^ 1u);
            put_v(t + 1, flags_next, buffer ^ 1u);
        }
        const int32_t i_after = t + 2 - t_begin;
        if ((i_after & 15) == 0) {
            known = known_from(i_after, pages_ahead);
            pages_ahead = pages_from(i_after + 16);
        }
        const uint32_t flags_after = flags_of(i_after);
        if (t + 2 < t_end) bring(i_after);

        // a wavefront whose rows see nothing of the tile has nothing to do
        if (flags & kSome) {
            f32x16 s[HT];
            TV x[kAhead];
            auto scores = [&](const f32x16 &from) {
                // The operands come out of the LDS several products ahead of their use.
#pragma unroll
                for (int i = 0; i < kAhead; i++) x[i] = k_operand(i, buffer);
#pragma unroll
                for (int i = 0; i < kProducts; i++) {
                    s[i / KS] = Mfma<T>::m32(x[i % kAhead], q[i % KS], i % KS ? s[i / KS] : from);
                    if (i + kAhead < kProducts) x[i % kAhead] = k_operand(i + kAhead, buffer);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
                for (int i = 0; i < kProducts - kAhead; i++) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);

                if (flags & kEdge) {
                    const int32_t j = first_token(t);
                    Seen here = seen;
                    here.high = min(here.high, end_of(flags));
#pragma unroll
                    for (int h = 0; h < HT; h++)
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            const int token = 32 * h + 8 * (i / 4) + i % 4; // of the lower half; the upper half's is 4 further, brought by the same wavefront
                            const bool sees = here.token(j + token + 4 * (int32_t)half) & ((flags >> (token / kTokens) & 1u) != 0);
                            s[h][i] = sees ? s[h][i] : -INFINITY;
                        }
                }
                float tops[4] = {s[0][0], s[0][1], s[0][2], s[0][3]}; // four chains of comparisons, not one of sixteen
#pragma unroll
                for (int i = 4; i < 16 * HT; i++) tops[i % 4] = fmaxf(tops[i % 4], s[i / 16][i % 16]);
                return max_over_32(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
            };
            // Scores come out of the products less a reference, with which the sums begin.  It moves, to the largest score so far, only when one
            // is so far above it that its weight would exceed 2^(kLiftMany + 8): weights stay inside the range of the type, and what has been
            // added up is scaled now and then, not for every tile.  Where it moves by more than 16 powers of two the products are made once more from
            // 0: a sum that began with a reference far below has lost the score's last bits, or all of them (64 keys with scores of -1e9
            // before ordinary ones).
            float top = scores(below);
            if (__any(top * a.scale > 8.0f || (!any && top != -INFINITY))) {
                const float old = -below[0]; // 0 if no score has been seen
                const bool again = __any(any && top * a.scale > 16.0f);
                if (again) top = scores(f32x16{});
                // by how much the scores go down, which are relative to the old reference or to 0
                const float shift = any ? fmaxf(top, again ? old : 0.0f) : top == -INFINITY ? 0.0f : top;
                const float next = again ? shift : old + shift;
                const float fade = any ? exp2_of((old - next) * a.scale) : 0.0f;
                any = any || top != -INFINITY;
                l *= fade;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[dt] *= fade;
#pragma unroll
                for (int h = 0; h < HT; h++) s[h] -= shift;
                below = f32x16{} - next;
            }
            TV w[kGroups];
#pragma unroll
            for (int i = 0; i < kAhead; i++) x[i] = v_operand(i, buffer);
#pragma unroll
            for (int u = 0; u < kGroups; u++) {
                typedef float f32x8 __attribute__((ext_vector_type(8)));
                auto lifted = [&](float x) { return Mfma<T>::kLiftMany == 0.0f ? x * a.scale : __builtin_fmaf(x, a.scale, Mfma<T>::kLiftMany); };
                f32x8 e;
#pragma unroll
                for (int i = 0; i < 8; i++) e[i] = exp2_of(lifted(s[u / 2][8 * (u % 2) + i]));
                l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                w[u] = __builtin_convertvector(e, TV);
            }
#pragma unroll
            for (int i = 0; i < kGroups * DT; i++) {
                o[i % DT] = Mfma<T>::m32(x[i % kAhead], w[i / DT], o[i % DT]);
                if (i + kAhead < kGroups * DT) x[i % kAhead] = v_operand(i + kAhead, buffer);
            }
            dcdev::in_register<false>(l); // the additions among the products, not behind them
            uint32_t odd_bits = 0;
            if (flags & kPartial) {
#pragma unroll
                for (int i = 0; i < 4; i++) odd_bits |= __builtin_amdgcn_readfirstlane(lds.odd[buffer][i]) << i;
            }
            if (odd_bits) {
#pragma unroll 1
                for (int i = 0; i < kTile; i++) {
                    const int32_t j = first_token(t);
                    if (!(odd_bits >> (i / kTokens) & 1u)) continue;
                    if (j + i >= end_of(flags)) continue;
                    const uint32_t place = (uint32_t)(j + i - (flags & kPrefix ? 0 : base));
                    const int32_t at = (flags & kPrefix ? prefix_table : own_table)[place >> a.batch.page_shift]; // there, or nothing of it would be odd
                    const T *src = static_cast<const T *>(a.v_pages) + (page_stride * (uint32_t)at + head_at + (place & place_mask)) * D + 4 * half;
                    const bool sees = seen.token(j + i);
#pragma unroll
                    for (int dt = 0; dt < DT; dt++)
#pragma unroll
                        for (int b = 0; b < 4; b++) {
                            f32x4 v = {o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]};
                            v = with_odd<T>(v, src + 32 * dt + 8 * b, sees);
                            o[dt][4 * b] = v[0], o[dt][4 * b + 1] = v[1], o[dt][4 * b + 2] = v[2], o[dt][4 * b + 3] = v[3];
                        }
                }
            }
        }
        flags = flags_next, flags_next = flags_after;
        __syncthreads();
    };

    if (t_begin < t_end) {
        flags = flags_of(0), flags_next = flags_of(1);
        bring(0);
        put_k(0);
        put_v(t_begin, flags, 0);
        if (t_begin + 1 < t_end) bring(1);
    }
    __syncthreads();
    for (int32_t t = t_begin; t < t_end; t += 2) {
        step(std::integral_constant<uint32_t, 0>{}, t);
        if (t + 1 < t_end) step(std::integral_constant<uint32_t, 1>{}, t + 1);
    }

    const f32x2 both = swapped32(l);
    const float total = both[0] + both[1];
    // what the weights are relative to (also if the row saw scores and none was a number)
    const float top = any || total != total ? -below[0] * a.scale - Mfma<T>::kLiftMany : -INFINITY;
    if (my_row >= n) return;
    uint32_t row = my_row; // where the results go is worked out here, not kept in registers from the beginning
    dcdev::anew(row);
    const uint32_t packed = row_first + row / a.group, head = kv * a.group + row % a.group;
    auto sums = [&](int dt, int b) { return f32x4{o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]}; };
    if (a.n_slots == 1) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        T *out = static_cast<T *>(a.out) + packed * a.out_row + head * a.out_head + 4 * half;
        const float r = 1.0f / total;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int b = 0; b < 4; b++) *reinterpret_cast<T4 *>(out + 32 * dt + 8 * b) = __builtin_convertvector(total == 0.0f ? f32x4{} : sums(dt, b) * r, T4);
        if (a.lse && half == 0) a.lse[(uint64_t)packed * a.n_heads + head] = total == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
    } else {
        const uint64_t i = ((uint64_t)packed * a.n_heads + head) * a.n_slots + part.first_slot + split;
        float *out = a.partial + i * D + 4 * half;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int b = 0; b < 4; b++) *reinterpret_cast<f32x4 *>(out + 32 * dt + 8 * b) = sums(dt, b);
        if (half == 0) a.partial_ml[i] = f32x2{top, total};
    }
}

template <int D> constexpr int workgroups_a_unit() { return D == 256 ? 1 : D == 64 ? 3 : 2; }
template <typename T, int D> __global__ __launch_bounds__(256, workgroups_a_unit<D>()) void dc_attention_tile_kernel(AttentionArgs a)
{
    __shared__ __align__(16) TileLds<D> lds;
    const bool common = blockIdx.x < a.prefix.blocks;
    many_rows<T, D>(a, lds, common, common ? blockIdx.x : blockIdx.x - a.prefix.blocks);
}

// A common prefix with many rows and few rows in each sequence: the first is bound by the matrix units, the second by memory, and the two
// kinds of workgroups lie in one launch in turn, so that a compute unit has some of each (64 sequences behind 16384 tokens: 67 us instead of 72
// in two launches; 62 since then, 5 of them the join).
// In turn by eights: a workgroup's XCD is its number modulo 8, and those of one key/value head's prefix stay on one.
template <typename T, int D, int RT> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void dc_attention_both_kernel(AttentionArgs a)
{
    __shared__ __align__(16) union {
        FewLds<D, RT> few;
        TileLds<D> many;
    } lds;
    const uint32_t eight = blockIdx.x >> 3, prefix_eights = (a.prefix.blocks + 7) / 8, own_eights = (a.own.blocks + 7) / 8, less = min(prefix_eights, own_eights);
    const bool common = eight < 2 * less ? (eight & 1u) == 0 : prefix_eights > own_eights;
    const uint32_t block = (eight < 2 * less ? eight / 2 : eight - less) * 8 + (blockIdx.x & 7u);
    if (common) {
        if (block < a.prefix.blocks) many_rows<T, D>(a, lds.many, true, block);
    } else {
        if (block < a.own.blocks) few_rows<T, D, RT>(a, lds.few, false, block);
    }
}

// Joins the splits of a row and head: each has its sums relative to a maximum of its own.  The weights of the splits first, into the LDS; then
// 4 D / 1024 of the threads go through every so many splits with several loads under way: 3 us for 32 rows and heads, 5.4 for 64 rows of 32 heads.  (The last
// split to arrive joining them all instead: every workgroup's device-wide fence empties its L2, one token 106 instead of 12 us.)
constexpr uint32_t kMostSplits = 128, kMostSlots = 2 * kMostSplits; // of a part, of both parts
template <typename T, int D> __global__ __launch_bounds__(256) void dc_attention_join_kernel(AttentionArgs a)
{
    constexpr uint32_t kQuads = D / 4, kSets = 256 / kQuads, kAtOnce = 4;
    __shared__ f32x4 lds_sum[kSets][kQuads];
    __shared__ float lds_weight[kMostSlots], lds_top[4], lds_total[4];
    const uint32_t row = blockIdx.x, head = blockIdx.y, at = threadIdx.x % kQuads, set = threadIdx.x / kQuads;
    const uint64_t first = ((uint64_t)row * a.n_heads + head) * a.n_slots;
    f32x2 ml = {-INFINITY, 0.0f};
    if (threadIdx.x < a.n_slots) ml = a.partial_ml[first + threadIdx.x];
    if (a.batch.sequence_of(row, a.max_new) >= a.batch.n_seqs) return;
    float top = max_over_16(ml[0]);
#pragma unroll
    for (int k = 1; k < 16; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    if ((threadIdx.x & 63u) == 0) lds_top[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(lds_top[0], lds_top[1]), fmaxf(lds_top[2], lds_top[3]));
    const float weight = ml[0] == -INFINITY ? 0.0f : exp2_of(ml[0] - top);
    lds_weight[threadIdx.x] = ml[0] == -INFINITY ? -1.0f : weight;
    float total = sum_over_16(ml[0] == -INFINITY ? 0.0f : ml[1] * weight);
#pragma unroll
    for (int k = 1; k < 16; k <<= 1) total += __shfl_xor(total, k);
    if ((threadIdx.x & 63u) == 0) lds_total[threadIdx.x >> 6] = total;
    __syncthreads();
    total = (lds_total[0] + lds_total[1]) + (lds_total[2] + lds_total[3]);
    f32x4 sum = {};
    const float *src = a.partial + first * D + 4 * at;
    for (uint32_t slot = set; slot < a.n_slots; slot += kSets * kAtOnce) {
        f32x4 v[kAtOnce];
        float w[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; i++) {
            const uint32_t k = slot + i * kSets;
            w[i] = k < a.n_slots ? lds_weight[k] : -1.0f; // a split that saw nothing has left nothing to add
            v[i] = f32x4{};
            if (w[i] >= 0.0f || w[i] != w[i]) v[i] = *reinterpret_cast<const f32x4 *>(src + (uint64_t)k * D);
        }
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; i++) sum += v[i] * w[i];
    }
    lds_sum[set][at] = sum;
    __syncthreads();
    if (set) return;
#pragma unroll
    for (uint32_t i = 1; i < kSets; i++) sum += lds_sum[i][at];
    store_whole<T>(a, row, head, 4 * at, sum, top, total);
}

// Which kernel works through a part: that for at most 16 rows or 32 rows, or that for many.
enum Kind { kFew16 = 0, kFew32 = 1, kTile = 2 };
struct Plan {
    Kind prefix_kind, own_kind;
};

bool attention_ok(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *t)
{
    if (!cache_ok(cache) || !batch_ok(cache, batch) || !t) return false;
    if ((uint64_t)batch->n_rows * t->n_heads >= 0x80000000ull) return false;
    if (t->n_heads < 1 || t->n_heads > 65535 || t->n_heads % cache->n_kv_heads) return false;
    if (!(fabsf(t->scale) <= 0x1p127f)) return false; // scale log2(e) is a number
    return t->q_dev && t->out_dev && t->q_dev != t->out_dev && aligned16(t->q_dev) && aligned16(t->out_dev) && ((uintptr_t)t->lse_dev & 3u) == 0 &&
           strides_ok(t->q_row_stride, t->q_head_stride) &&
           strides_apart(t->out_row_stride, t->out_head_stride, batch->n_rows, t->n_heads, cache->head_dim);
}

template <typename T, int D> void launch(const AttentionArgs &a, const Plan &plan, hipStream_t stream)
{
    const dim3 threads(256);
    if (a.prefix.blocks && plan.prefix_kind == kTile && plan.own_kind != kTile) {
        const dim3 grid(8 * ((a.prefix.blocks + 7) / 8 + (a.own.blocks + 7) / 8));
        if (plan.own_kind == kFew16) hipLaunchKernelGGL((dc_attention_both_kernel<T, D, 1>), grid, threads, 0, stream, a);
        else if constexpr (D < 256) hipLaunchKernelGGL((dc_attention_both_kernel<T, D, 2>), grid, threads, 0, stream, a);
    } else { // a sequence's rows are never more than the batch's: both parts are of the kind of their rows together, or the prefix is alone
        const Kind kind = a.prefix.blocks ? std::max(plan.prefix_kind, plan.own_kind) : plan.own_kind;
        const dim3 grid(a.prefix.blocks + a.own.blocks);
        if (kind == kFew16) hipLaunchKernelGGL((dc_attention_few_kernel<T, D, 1>), grid, threads, 0, stream, a);
        else if (kind == kTile) hipLaunchKernelGGL((dc_attention_tile_kernel<T, D>), grid, threads, 0, stream, a);
        else if constexpr (D < 256) hipLaunchKernelGGL((dc_attention_few_kernel<T, D, 2>), grid, threads, 0, stream, a);
    }
    if (a.n_slots > 1)
        hipLaunchKernelGGL((dc_attention_join_kernel<T, D>), dim3(a.batch.n_rows, a.n_heads), threads, 0, stream, a);
}

template <typename T> void launch_d(const AttentionArgs &a, const Plan &plan, uint32_t head_dim, hipStream_t stream)
{
    if (head_dim == 64) launch<T, 64>(a, plan, stream);
    else if (head_dim == 128) launch<T, 128>(a, plan, stream);
    else launch<T, 256>(a, plan, stream);
}

// How a call's keys are cut: fills prefix, own and n_slots, and gives the bytes of workspace.  False for a batch that is too large.
bool make_plan(AttentionArgs &a, Plan &plan, const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *t, uint64_t *workspace_bytes)
{
    *workspace_bytes = 0;
    const uint64_t group = t->n_heads / cache->n_kv_heads, d = cache->head_dim, prefix_len = batch->prefix_len;
    // Up to 32 rows the kernel for few rows, of the matrix units' 16 or 32 (16 sequences of 8192 tokens, 8 heads of 128: 16 rows 88 us, by the kernel
    // for many 119; 20 rows 91 and 122; of one sequence, 16 rows of 4000 tokens 11.5 and 13.9, but 20 rows of 8192 19.1 and 16.4).  Heads of
    // 256 have no registers for 32.
    auto kind_of = [&](uint64_t rows) { return rows <= 16 ? kFew16 : rows <= 32 && d < 256 ? kFew32 : kTile; };
    const uint64_t all_rows = batch->n_rows * group, seq_rows = batch->max_new * group;
    const Kind prefix_kind = kind_of(all_rows), own_kind = kind_of(seq_rows);
    plan = Plan{prefix_kind, own_kind};
    const uint64_t own_len = batch->max_len > prefix_len ? batch->max_len - prefix_len : 1;
    const uint64_t seq_tiles = (seq_rows + kTileRows - 1) / kTileRows; // workgroups to a sequence's rows
    // upper bound of the workgroups' number, as the kernel counts them off
    const uint64_t row_tiles = !batch->row_start_dev ? batch->n_seqs * seq_tiles : std::min<uint64_t>(all_rows / kTileRows + batch->n_seqs, all_rows);
    const uint64_t tile_many = d == 256 ? 32 : 64;
    const double unit_rate = d == 64 ? 1.5 : d == 128 ? 0.87 : 0.55; // steps a us of a full compute unit in the kernel for many rows

    // Of the kernel for few rows: items are workgroups uncut.
    auto cut_few = [&](uint64_t items, uint64_t tokens) {
        constexpr uint64_t tile = 32, least = 4;
        const uint64_t n_tiles = (tokens + tile - 1) / tile, most = std::max<uint64_t>(1, std::min<uint64_t>((n_tiles + least - 1) / least, kMostSplits));
        // Up to three tiles to a wavefront, parts gain less than it costs to join them (8 heads, 200 tokens: 6.9 us, in parts 8.5; 400: 9.0 and 8.7).
        if (!prefix_len && n_tiles <= 12) return (uint64_t)1;
        uint64_t n = 1;
        // As few workgroups as give every compute unit the same number, to a tenth: a long run of keys is read faster by one workgroup
        // (256 of 8 heads' and 32 sequences' runs of 8000 tokens: 161 us, 512 halves of them 168, 1024 quarters 176), but an uneven number
        // leaves units idle (320 runs of 4100 tokens: 124 us, 960 thirds 108).
        while (n < most && (items * n + 255) / 256 * 256 * 10 > items * n * 11) n++;
        // Where little is to be read, its latency counts: two workgroups to a unit (one token over 1999, 32 heads: 12.0 us with 256, 11.6 with 512).
        if (!prefix_len && items * n <= 256 && (n_tiles + n - 1) / n <= 16) n = std::min(2 * n, most);
        return n;
    };
    // Of the kernel for many rows: the number of parts with the least estimate of the time, in us.  A tile's step takes `step` where a workgroup
    // has its compute unit to itself, and a unit does unit_rate steps a us where it is full; joining costs a launch and the parts' way to
    // memory and back.
    auto cut_many = [&](uint64_t items, uint64_t tokens, uint64_t fewer_tokens, bool joined_anyway) {
        const double tile = tile_many, step = d == 64 ? 1.2 : d == 128 ? 1.4 : 1.8;
        const double most = std::max(1.0, ceil(tokens / tile)), mean = std::max(1.0, (tokens + fewer_tokens) / 2 / tile);
        uint64_t best = 1;
        double least = 1e30;
        for (uint64_t n = 1; n <= std::min<uint64_t>((uint64_t)most, kMostSplits); n += n < 8 ? 1 : n / 4) {
            const double join = n > 1 || joined_anyway ? 4 + all_rows * cache->n_kv_heads * n * (8e-6 * d) / (joined_anyway ? 2 : 4) : 0;
            const double time = std::max(ceil(most / n) * std::max(step, ceil(items * n / 256.0) / unit_rate), items * mean / (256 * unit_rate)) + join;
            if (time < least) least = time, best = n;
        }
        return best;
    };
    auto part = [&](uint64_t items, uint64_t tokens, uint64_t tile, uint64_t n, uint32_t first_slot) {
        const uint64_t n_tiles = std::max<uint64_t>(1, (tokens + tile - 1) / tile), chunk = (n_tiles + n - 1) / n;
        n = (n_tiles + chunk - 1) / chunk;
        return items * n < 1u << 24 ? Part{(uint32_t)(items * n), (uint32_t)n, (uint32_t)chunk, first_slot} : Part{};
    };
    // what a row, or some rows together, can see
    auto seen = [&](uint64_t tokens, uint64_t rows) { return t->window ? std::min(tokens, (uint64_t)t->window + rows + t->sinks + 64) : tokens; };
    // a sequence's many rows, over their own pages or over the prefix along with them
    auto many_part = [&](bool along) {
        const uint64_t longest = along ? prefix_len + own_len : own_len, rows = kTileRows / group + 1;
        const uint64_t tokens = seen(longest, rows), fewer = seen(longest > batch->max_new ? longest - batch->max_new : 1, rows);
        const uint64_t filled = std::max<uint64_t>(1, all_rows / kTileRows); // of the workgroups counted off, about
        return part(cache->n_kv_heads * row_tiles, tokens, tile_many, cut_many(cache->n_kv_heads * filled, tokens, fewer, a.prefix.blocks != 0), a.prefix.n_splits);
    };
    // A sequence's many rows read the prefix along with their own pages where that is estimated to cost less than to read it once for all sequences' rows
    // together and to join the two.  It costs the steps of the workgroups that it takes beyond those of all rows together, of the prefix only what
    // the middle one of the longest sequence's rows sees through the window; and it saves the join, or part of it where what it takes is itself
    // cut and joined.  The two constants beside the measured rates (0.8; 0.4) are fitted to both ways' times at 64 sizes: the slower way is taken
    // at 3 of them, by 12, 1.3 and 0.6 %.  Heads of 128, 8 of keys and values (us; read along, and once): 8 sequences of 64 rows behind 512 tokens 19 and
    // 23, behind 4096 32.5 and 30.8; of 160 rows 23 and 33, 65 and 56; of 400 behind 4096 97 and 106, behind 16384 297 and 270; 64 sequences of
    // 36 rows behind 512 40 and 66, behind 16384 500 and 208, there with a window of 12000 371 and 163, of 1500 54 and 68.
    if (prefix_len && own_kind == kTile) {
        const Part along = many_part(true);
        const uint64_t shared_tiles = (all_rows + kTileRows - 1) / kTileRows;
        const uint64_t more_tiles = batch->n_seqs * seq_tiles - std::min(batch->n_seqs * seq_tiles, shared_tiles);
        const int64_t behind = (int64_t)own_len - (int64_t)(batch->max_new + 1) / 2;
        const uint64_t prefix_seen = t->window ? std::min<uint64_t>(prefix_len, std::max<int64_t>((int64_t)t->window - behind, 0) + t->sinks) : prefix_len;
        const double more_time = 0.8 * more_tiles * cache->n_kv_heads * prefix_seen / tile_many / (256 * unit_rate);
        const double parts_time = all_rows * cache->n_kv_heads * (8e-6 * d);
        const double join_time = 4 + parts_time - (along.n_splits > 1 ? 0.4 * (4 + parts_time * along.n_splits / 4) : 0.0);
        a.whole = along.blocks && more_time <= join_time;
        if (a.whole) a.own = along;
    }
    if (prefix_len && !a.whole) {
        const uint64_t tokens = seen(prefix_len, batch->max_new);
        if (prefix_kind == kTile) {
            const uint64_t items = cache->n_kv_heads * ((all_rows + kTileRows - 1) / kTileRows);
            a.prefix = part(items, tokens, tile_many, cut_many(items, tokens, tokens, true), 0);
        } else {
            a.prefix = part(cache->n_kv_heads, tokens, 32, cut_few(cache->n_kv_heads, tokens), 0);
        }
        if (!a.prefix.blocks) return false;
    }
    if (own_kind == kTile) {
        if (!a.whole) a.own = many_part(false);
    } else {
        const uint64_t tokens = seen(own_len, batch->max_new), items = (uint64_t)cache->n_kv_heads * batch->n_seqs;
        a.own = part(items, tokens, 32, cut_few(items, tokens), a.prefix.n_splits);
    }
    if (!a.own.blocks || (uint64_t)a.own.blocks + a.prefix.blocks >= 1u << 24) return false;
    a.n_slots = a.prefix.n_splits + a.own.n_splits;
    if (a.n_slots > 1) *workspace_bytes = (uint64_t)batch->n_rows * t->n_heads * a.n_slots * (d + 2) * sizeof(float);
    return true;
}

} // namespace

extern "C" int dc_attention_paged_workspace(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *attention,
                                            uint64_t *workspace_bytes)
{
    if (!workspace_bytes || !attention_ok(cache, batch, attention)) return DC_E_ARG;
    AttentionArgs a = {};
    Plan plan;
    return make_plan(a, plan, cache, batch, attention, workspace_bytes) ? DC_OK : DC_E_ARG;
}

extern "C" int dc_attention_paged(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *attention,
                                  void *workspace_dev, uint64_t workspace_bytes, void *hip_stream)
{
    if (!attention_ok(cache, batch, attention) || !aligned16(workspace_dev)) return DC_E_ARG;
    AttentionArgs a = {};
    a.batch = batch_args(cache, batch);
    a.k_pages = cache->k_dev, a.v_pages = cache->v_dev, a.q = attention->q_dev, a.out = attention->out_dev, a.lse = attention->lse_dev;
    a.q_row = attention->q_row_stride, a.q_head = attention->q_head_stride;
    a.out_row = attention->out_row_stride, a.out_head = attention->out_head_stride;
    a.n_heads = attention->n_heads, a.n_kv_heads = cache->n_kv_heads, a.group = a.n_heads / a.n_kv_heads;
    a.window = attention->window, a.sinks = attention->sinks, a.max_new = batch->max_new;
    a.negate = attention->scale < 0.0f;
    // Never 0, which would turn the -infinity of hidden tokens into NaN: the smallest number that there is leaves of any score less than 2^-21.
    a.scale = std::max(fabsf(attention->scale) * kLog2e, 0x1p-149f);
    uint64_t needed = 0;
    Plan plan;
    if (!make_plan(a, plan, cache, batch, attention, &needed) || (needed && !workspace_dev)) return DC_E_ARG;
    if (workspace_bytes < needed) return DC_E_CAP;
    a.partial = static_cast<float *>(workspace_dev);
    a.partial_ml = reinterpret_cast<f32x2 *>(a.partial + (uint64_t)batch->n_rows * a.n_heads * a.n_slots * cache->head_dim);
    if (cache->type == DC_TYPE_BF16) launch_d<__bf16>(a, plan, cache->head_dim, static_cast<hipStream_t>(hip_stream));
    else launch_d<_Float16>(a, plan, cache->head_dim, static_cast<hipStream_t>(hip_stream));
    return dc_launch_status();
}
