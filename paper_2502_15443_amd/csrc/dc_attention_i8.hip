// Attention of new tokens over a paged cache of keys and values held in 8 bits: whole numbers times a scale for each block of tokens of a head.
//
// For a row with query q: s_j = scale ks_j (q . k_j), out = sum_j exp(s_j - m) vs_j v_j / sum_j exp(s_j - m) with the running maximum m, where k_j and
// v_j are the whole numbers and ks_j, vs_j their blocks' scales.  The numbers are exact in f16: products are the matrix units' f16 ones, also of bf16 queries;
// a key's scale is put on the sum, a value's scale on the weight before its product.  A hidden token's numbers are numbers, whatever the cache holds: a weight of
// 0 keeps it out.
#include "dc_attention.h"

#include <algorithm>

using namespace dcattn;

namespace {

// 4 whole numbers of 8 bits in f16: with its sign bit turned a byte is 128 more, as the low byte of an f16 between 1024 and 2048 it is exact, and less 1152 it is
// the number.  5 operations; conversions byte by byte take 6.
__device__ __forceinline__ u32x2 four_f16(uint32_t x)
{
    const uint32_t more = x ^ 0x80808080u;
    const f16x2 less = {(_Float16)1152.0f, (_Float16)1152.0f};
    const f16x2 low = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, more, 0x04010400u)) - less;
    const f16x2 high = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, more, 0x04030402u)) - less;
    return u32x2{__builtin_bit_cast(uint32_t, low), __builtin_bit_cast(uint32_t, high)};
}
__device__ __forceinline__ u32x4 eight_f16(uint32_t x, uint32_t y)
{
    const u32x2 a = four_f16(x), b = four_f16(y);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// Of 8 rows of 16 values of 8 bits that the 16 lanes name (half a row each), lane i gets column i.
__device__ __forceinline__ u32x2 lds_column8(uint32_t addr)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(uintptr_t)addr));
}

// Queries as f16.  Those of bf16 are brought to a largest one of 2^14 to 2^15 by a power of two, of which the score gets the reciprocal: the 8 bits of
// all that are above 2^-29 times the largest stay as they are, and those below are off by 2^-40 of it at most, far less than the sum's own roundings.
// `most`: largest of the row's values, as bits without sign.
template <typename T> struct Queries;
template <> struct Queries<_Float16> {
    float back = 1.0f;
    __device__ __forceinline__ explicit Queries(uint32_t) {}
    __device__ __forceinline__ f16x8 operator()(u32x4 x) const { return __builtin_bit_cast(f16x8, x); }
};
template <> struct Queries<__bf16> {
    float by, back;
    __device__ __forceinline__ explicit Queries(uint32_t most)
    {
        const uint32_t e = min(268u - (most >> 7), 253u); // 2^(e - 127): reciprocals are numbers too
        by = __uint_as_float(e << 23), back = __uint_as_float((254u - e) << 23);
    }
    __device__ __forceinline__ f16x8 operator()(u32x4 x) const
    {
        return __builtin_convertvector(__builtin_convertvector(__builtin_bit_cast(bf16x8, x), f32x8) * by, f16x8);
    }
};
// Largest of 16-bit values without their signs.
__device__ __forceinline__ uint32_t largest(uint32_t m, const u32x4 &x)
{
    u16x2 v = {(uint16_t)m, 0};
#pragma unroll
    for (int i = 0; i < 4; i++) v = __builtin_elementwise_max(v, __builtin_bit_cast(u16x2, x[i] & 0x7FFF7FFFu));
    return max((uint32_t)v[0], (uint32_t)v[1]);
}

// Largest over the lanes with the same number modulo 16 (32).
__device__ __forceinline__ uint32_t largest_over_32(uint32_t v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t largest_over_16(uint32_t v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return largest_over_32(max(r[0], r[1]));
}

// Weights go into the product with the values as f16, times the value's scale over the largest scale of a block that the row has seen a token of, rounded up to a
// power of two.  f16 loses bits below 2^-14 and everything below 2^-25, and its largest value is 2^16: the exponentials' reference lies kLift below the largest
// score, so that the largest weight is 2^15 in the kernel for few rows and 2^7 to 2^15 in the one for many.
constexpr int kLiftFew = 15, kLiftMany = 7;
struct ValueScale {
    uint32_t ref = 0, least = 0; // of the lane's row: bits of that scale; the smallest of the wavefront's rows
    float by = 0.0f;             // 1 / ref
    // (one of a row that is not there never has to grow)
    __device__ __forceinline__ void begin(bool there) { set(there ? 1u << 23 : 254u << 23); }
    __device__ __forceinline__ float value() const { return __uint_as_float(ref); }
    // A scale over it: 1 at most, and for a scale of tokens that the row does not see, whose weights are 0, anything up to 1.
    __device__ __forceinline__ float share(float scale) const { return __builtin_amdgcn_fmed3f(scale * by, 0.0f, 1.0f); }
    __device__ __forceinline__ static uint32_t power_above(uint32_t scale_bits) { return (scale_bits + 0x7FFFFFu) & 0x7F800000u; }
    // Whether the row's has to grow if it sees a scale; whether that of any row would have to, by a scalar comparison (in the kernel for few rows 64 sequences of up to 8192
    // tokens 120.9 us, by the lanes' 122.4; in the one for many, where some row mostly sees none of the tokens yet, pieces behind a window 70.1 and 69.0).
    __device__ __forceinline__ bool below(uint32_t scale_bits) const { return power_above(scale_bits) > ref; }
    __device__ __forceinline__ bool may_grow(uint32_t most_bits) const { return power_above(most_bits) > least; }
    // Takes in the largest scale that the row sees; by what its sums are multiplied then.
    __device__ __forceinline__ float take_in(uint32_t scale_bits)
    {
        const uint32_t before = ref;
        set(max(power_above(scale_bits), ref));
        return __uint_as_float((uint32_t)max((int32_t)((127u << 23) + before - ref), 0));
    }

private:
    __device__ __forceinline__ void set(uint32_t bits)
    {
        ref = bits, by = __uint_as_float(max((254u << 23) - bits, 0x400000u)); // (1 / 2^127 is below the normal range)
        least = ~largest_of_lanes(~bits);
    }
};

// ---- few rows -------------------------------------------------------------------------------------------------------------
//
// At most 16 RT rows (new tokens times the query heads that share a key/value head) read the keys: memory bounds this kernel.  A
// wavefront takes tiles of 64 tokens.  Scores come as a matrix [token][row] = K Q^T, of which a lane holds 4 tokens of one row in each quarter of
// the tile; two quarters are the second operand of [head_dim][row] = V^T P^T if the product's 32 tokens are numbered that way.  K and then V go through
// registers into the wavefront's own part of the LDS, as bytes, and become f16 on their way to the products: of K a lane reads 16 neighbouring values of a
// token, for two products; of V the transposing read gives it 8 tokens of one value.  No barrier in the loop; the next tile's loads are under way during the
// rest of the tile's work.  64 sequences of 4096 tokens, 32 heads on 8 of 128: 88 us, 6.1 TB/s; where lengths differ by up to 16, 121 us, 4.9 TB/s, for
// sequences end at unlike times (shares of equal length, cut on the device: 118 to 126, the alike ones 93 to 103); one of 131071 tokens 52 us.  A tile of 64
// tokens takes 590 vector operations and 210 registers, for two workgroups a compute unit (three, of 168, spill: 84 us).
template <int D, int RT> struct FewLds {
    static constexpr int kPadded = D + 4; // floats of a row's sums
    union {
        uint8_t tokens[4][few_tile(RT) * D]; // of each wavefront: a tile's keys, then its values
        float sums[4][16][kPadded];
    };
    float m[4][16 * RT], l[4][16 * RT];
    int32_t p[16 * RT];
};

// APART: the parts of these rows are theirs alone.
template <typename T, int D, int RT, bool APART = false> __device__ __forceinline__ void few_rows(const AttentionArgs &a, const Part &part, FewLds<D, RT> &lds, bool common, uint32_t item)
{
    constexpr int kTile = few_tile(RT), kQuarters = kTile / 16, KS = D / 32, DT = D / 16;
    constexpr int kChunks = D / 16, kTokensALoad = 64 / kChunks, kLoads = kTile / kTokensALoad; // chunks: of 16 bytes

    // (a workgroup may have two of these, of 256 threads each)
    const uint32_t thread = threadIdx.x & 255u, lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(thread >> 6), c = lane & 15u, g = lane >> 4;
    const uint32_t kv = item % a.n_kv_heads;
    item /= a.n_kv_heads;
    const uint32_t seq = common ? 0 : item % a.batch.n_seqs, split = common ? item : item / a.batch.n_seqs;
    const int32_t *table = common ? a.batch.prefix_pages : a.batch.pages + (uint64_t)seq * a.batch.pages_stride;
    const uint32_t table_entries = common ? (a.batch.prefix_len + (1u << a.batch.page_shift) - 1) >> a.batch.page_shift : a.batch.pages_stride;
    // the table's entry of 16 tokens of a tile, in each lane that of the 16 with its number modulo kQuarters
    auto entry_at = [&](uint32_t j) {
        const uint32_t i = (j + 16 * (lane % kQuarters)) >> a.batch.page_shift;
        return i < table_entries ? table[i] : -1;
    };
    // Without a window it is known at once where a wavefront's first tile is: its pages are asked for together with the sequence's length.
    int32_t first_entry = -1;
    const uint64_t first_tile = (uint64_t)split * part.chunk + wave;
    if (!a.window && first_tile < 0x80000000u / kTile) first_entry = entry_at((uint32_t)first_tile * kTile);

    // rows of this workgroup: row_first + i / group of head kv * group + i % group for i < n
    uint32_t row_first = 0, n;
    int32_t p_first = 0, there, base = 0, p_min, p_max;
    if (common) {
        n = a.batch.n_rows * a.group;
        there = (int32_t)a.batch.prefix_len;
        // positions of the rows, sequence by sequence
        if (thread < 16 * RT) lds.p[thread] = kNoPosition;
        __syncthreads();
        for (uint32_t b = thread; b < a.batch.n_seqs; b += 256) {
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
        if (n > 16 * RT) return; // it is among those with many rows
        base = (int32_t)a.batch.prefix_len;
        there = min(max(len - base, 0), (int32_t)(a.batch.pages_stride << a.batch.page_shift));
        p_first = len - (int32_t)(end - row_first);
        p_min = p_first - base, p_max = p_first + (int32_t)rows - 1 - base;
    }
    const Tiles<kTile> tiles(p_min, p_max, there, a.window, (int64_t)a.sinks - base);
    const int32_t t_begin = (int32_t)min((uint64_t)split * part.chunk, (uint64_t)tiles.count);
    const int32_t t_end = split + 1 == part.n_splits ? tiles.count : (int32_t)min((uint64_t)t_begin + part.chunk, (uint64_t)tiles.count);

    // queries, and what the lane's rows see
    f16x8 q[RT][KS];
    ValueScale value_scale[RT];
    float row_scale[RT]; // with a key's scale it makes powers of two of the scores as they come out of the products
    Seen seen[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const uint32_t r = rt * 16 + c;
        const bool is = r < n;
        const uint32_t i = r / a.group, head = kv * a.group + r % a.group;
        seen[rt] = Seen(!is ? kNoPosition : common ? lds.p[i] : p_first + (int32_t)i - base, there, a.window, (int64_t)a.sinks - base);
        // of 64 neighbouring values the lane has 16, for two products: as it has of a key's
        const T *src = static_cast<const T *>(a.q) + (uint64_t)(row_first + i) * a.q_row + head * a.q_head + 16 * g;
        u32x4 x[KS];
        uint32_t most = 0;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            x[s] = u32x4{};
            if (is) x[s] = *reinterpret_cast<const u32x4 *>(src + 64 * (s / 2) + 8 * (s % 2));
            if (a.negate) x[s] ^= 0x80008000u;
            most = largest(most, x[s]);
        }
        value_scale[rt].begin(is);
        const Queries<T> as_f16(largest_over_16(most));
        row_scale[rt] = fminf(fmaxf(a.scale * as_f16.back, 0x1p-149f), 0x1p127f);
#pragma unroll
        for (int s = 0; s < KS; s++) q[rt][s] = as_f16(x[s]);
    }

    f32x4 o[RT][DT];
    float m[RT], l[RT]; // what a row's weights are relative to, kLiftFew below its largest score; their sum
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        m[rt] = -INFINITY, l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) o[rt][dt] = f32x4{};
    }

    const uint64_t page_stride = (uint64_t)a.n_kv_heads << a.batch.page_shift; // in tokens of a head
    const uint64_t head_at = (uint64_t)kv << a.batch.page_shift;
    const uint32_t place_mask = (1u << a.batch.page_shift) - 1u;
    auto page_from = [&](int32_t entry) { return (uint32_t)entry < a.batch.n_pages ? entry : -1; };
    auto page_of = [&](int32_t page, int quarter) { return __builtin_amdgcn_readlane(page, quarter); };
    // Scales of a tile: the first kQuarters lanes have those of the keys, the next ones those of the values; 16 tokens are inside a block.
    const float *scales = lane & kQuarters ? a.v_scales : a.k_scales;
    // Of tokens that no row sees they may be anything.
    auto sound_of = [&](int32_t j, int32_t page, float scale) {
        const int32_t first = j + 16 * (int32_t)(lane % kQuarters);
        const bool some = (page >= 0) & (first < tiles.high) & ((first + 16 > tiles.low) | (first < tiles.sinks));
        return some ? sound_scale(scale) : 0x1p-126f;
    };
    auto scale_of = [&](int32_t j, int32_t page) {
        const uint64_t at = (((uint64_t)(uint32_t)max(page, 0) * a.n_kv_heads + kv) << (a.batch.page_shift - a.block_shift)) +
                            ((((uint32_t)j + 16 * (lane % kQuarters)) & place_mask) >> a.block_shift);
        return scales[at];
    };
    u32x4 k[kLoads], v[kLoads];
    // A tile's keys or values in the order of memory, whole tokens side by side; nothing else will ask for them.  Where there is no page, those of page 0, which
    // are then taken for hidden.
    auto load = [&](u32x4 (&to)[kLoads], const void *pages, int32_t j, int32_t page) {
#pragma unroll
        for (int h = 0; h < kQuarters; h++) {
            const uint64_t first = page_stride * (uint32_t)max(page_of(page, h), 0) + head_at + ((uint32_t)(j + 16 * h) & place_mask);
            const uint8_t *src = static_cast<const uint8_t *>(pages) + first * D + lane * 16;
#pragma unroll
            for (int i = 0; i < kLoads / kQuarters; i++) to[h * (kLoads / kQuarters) + i] = dcdev::load16_stream(src + i * 1024);
        }
    };
    // Tokens lie in the LDS with their 16-byte chunks exchanged so that 16 tokens' same chunks are on different banks.
    auto swizzle = [](uint32_t token) { return D == 64 ? token >> 2 & 3u : D == 128 ? token >> 1 & 7u : token & 15u; };
    const uint32_t my_lds = dcdev::lds_address(lds.tokens[wave]);
    auto put = [&](const u32x4 (&from)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t token = i * kTokensALoad + lane / kChunks, chunk = lane % kChunks;
            *(lds_u32x4 *)(uintptr_t)(my_lds + token * D + ((chunk ^ swizzle(token)) << 4)) = from[i];
        }
        __builtin_amdgcn_wave_barrier();
    };

    // of this tile and the next one: pages of the quarters, scales; of the one behind it the table's entries
    int32_t page = -1, next_page = -1, entry = -1;
    float scale = 0.0f, next_scale = 0.0f;
    int32_t t = t_begin + (int32_t)wave;
    auto token_of = [&](int32_t t) { return tiles.first_token(min(t, t_end - 1)); };
    if (t < t_end) {
        const int32_t j = token_of(t);
        page = page_from(a.window ? entry_at((uint32_t)j) : first_entry);
        next_page = page_from(entry_at((uint32_t)token_of(t + 4)));
        scale = scale_of(j, page);
        load(k, a.k_pages, j, page);
        load(v, a.v_pages, j, page);
        entry = entry_at((uint32_t)token_of(t + 8));
    }
    for (; t < t_end; t += 4) {
        const int32_t j = token_of(t), next_j = token_of(t + 4);
        const bool more = t + 4 < t_end;

        put(k);
        if (more) {
            next_scale = scale_of(next_j, next_page);
            load(k, a.k_pages, next_j, next_page);
        }
        const float sound = sound_of(j, page, scale);
        auto scale_in = [&](int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(sound), lane)); };
        f32x4 s[RT][kQuarters];
#pragma unroll
        for (int h = 0; h < kQuarters; h++) {
#pragma unroll
            for (int rt = 0; rt < RT; rt++) s[rt][h] = f32x4{};
#pragma unroll
            for (int i = 0; i < KS / 2; i++) {
                const uint32_t token = 16 * h + c, chunk = 4 * i + g;
                const u32x4 x = *(const lds_u32x4 *)(uintptr_t)(my_lds + token * D + ((chunk ^ swizzle(token)) << 4));
                const f16x8 low = __builtin_bit_cast(f16x8, eight_f16(x[0], x[1])), high = __builtin_bit_cast(f16x8, eight_f16(x[2], x[3]));
#pragma unroll
                for (int rt = 0; rt < RT; rt++) {
                    s[rt][h] = Mfma<_Float16>::m16(low, q[rt][2 * i], s[rt][h]);
                    s[rt][h] = Mfma<_Float16>::m16(high, q[rt][2 * i + 1], s[rt][h]);
                }
            }
            const float ks = scale_in(h);
#pragma unroll
            for (int rt = 0; rt < RT; rt++) s[rt][h] *= fminf(ks * row_scale[rt], 0x1p127f); // powers of two from here on
        }
        __builtin_amdgcn_wave_barrier();
        put(v);
        if (more) load(v, a.v_pages, next_j, next_page);

        // tokens that not all rows see
        const bool edge = __any(page < 0) || j + kTile > p_min + 1 || j + kTile > tiles.high || (j < tiles.low && j + kTile > tiles.sinks) ||
                          (a.window && j + kTile > tiles.sinks && (int64_t)j <= (int64_t)p_max - a.window);
        float vs[kQuarters];
        uint32_t most_vs = 0;
#pragma unroll
        for (int h = 0; h < kQuarters; h++) vs[h] = scale_in(kQuarters + h), most_vs = max(most_vs, __float_as_uint(vs[h]));
        f16x8 w[RT][kQuarters / 2];
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            uint32_t row_vs = most_vs; // of what the row sees
            if (edge) {
                row_vs = 0;
#pragma unroll
                for (int h = 0; h < kQuarters; h++) row_vs = max(row_vs, seen[rt].some_of16(j + 16 * h) ? __float_as_uint(vs[h]) : 0u);
#pragma unroll
                for (int h = 0; h < kQuarters; h++) {
                    const bool is_there = page_of(page, h) >= 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool sees = seen[rt].token(j + 16 * h + 4 * (int32_t)g + i) & is_there;
                        s[rt][h][i] = sees ? s[rt][h][i] : -INFINITY;
                    }
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < kQuarters; h++) top = fmaxf(top, fmaxf(fmaxf(s[rt][h][0], s[rt][h][1]), fmaxf(s[rt][h][2], s[rt][h][3])));
            if (value_scale[rt].may_grow(most_vs)) {
                const float less = value_scale[rt].take_in(row_vs);
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[rt][dt] *= less;
            }
            top = fmaxf(m[rt], max_over_16(top) - kLiftFew);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float fade = exp2_of(m[rt] - ref);
            m[rt] = top;
            float sum = 0.0f;
#pragma unroll
            for (int u = 0; u < kQuarters / 2; u++) {
                f32x8 e;
#pragma unroll
                for (int i = 0; i < 8; i++) e[i] = exp2_of(s[rt][2 * u + i / 4][i % 4] - ref);
                sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                const float share[2] = {value_scale[rt].share(vs[2 * u]), value_scale[rt].share(vs[2 * u + 1])};
#pragma unroll
                for (int i = 0; i < 8; i++) e[i] *= share[i / 4];
                w[rt][u] = __builtin_convertvector(e, f16x8);
            }
            l[rt] = l[rt] * fade + sum;
#pragma unroll
            for (int dt = 0; dt < DT; dt++) o[rt][dt] *= fade;
        }
        // of 32 tokens the lane's group of 16 has 4 of each of two quarters, as the weights are
        const uint32_t i8 = c >> 1, token8 = 4 * g + (i8 & 3u) + (i8 >> 2) * 16;
#pragma unroll
        for (int u = 0; u < kQuarters / 2; u++)
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
                const uint32_t token = token8 + 32 * u;
                const u32x2 x = lds_column8(my_lds + token * D + (((uint32_t)dt ^ swizzle(token)) << 4) + ((c & 1u) << 3));
                const f16x8 values = __builtin_bit_cast(f16x8, eight_f16(x[0], x[1]));
#pragma unroll
                for (int rt = 0; rt < RT; rt++) o[rt][dt] = Mfma<_Float16>::m16(values, w[rt][u], o[rt][dt]);
            }
        __builtin_amdgcn_wave_barrier();
        page = next_page, scale = next_scale;
        next_page = page_from(entry);
        if (more) entry = entry_at((uint32_t)token_of(t + 12));
    }

    // the wavefronts' sums, brought to one maximum and added up in their order
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        l[rt] = sum_over_16(l[rt]) * __uint_as_float((127u - kLiftFew) << 23), m[rt] += kLiftFew;
        if (l[rt] != l[rt] && m[rt] == -INFINITY) m[rt] = 0.0f; // saw scores, none of them a number
        if (g == 0) lds.m[wave][rt * 16 + c] = m[rt], lds.l[wave][rt * 16 + c] = l[rt];
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const uint32_t r = rt * 16 + c;
        const float top = fmaxf(fmaxf(lds.m[0][r], lds.m[1][r]), fmaxf(lds.m[2][r], lds.m[3][r]));
        // (the largest scale, and what the weights were lifted by, in two steps: neither product leaves the range)
        const float f = m[rt] == -INFINITY ? 0.0f : exp2_of(m[rt] - top - kLiftFew) * value_scale[rt].value();
        if (rt) __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
            *reinterpret_cast<f32x4 *>(&lds.sums[wave][c][16 * dt + 4 * g]) = m[rt] == -INFINITY ? f32x4{} : o[rt][dt] * f;
        __syncthreads();
        constexpr uint32_t kQuads = D / 4;
        for (uint32_t i = thread; i < 16 * kQuads; i += 256) {
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
            const uint32_t in_seq = rr / a.group, head = kv * a.group + rr % a.group;
            if (!APART) {
                store_result<T, D>(a, row_first + in_seq, head, part.first_slot + split, at, sum, big, total);
            } else if (part.n_splits == 1) {
                store_whole<T>(a, row_first + in_seq, head, at, sum, big, total);
            } else {
                const uint64_t to = (((uint64_t)seq * a.few_rows_a_seq + in_seq) * a.n_heads + head) * part.n_splits + split;
                *reinterpret_cast<f32x4 *>(a.few_partial + to * D + at) = sum;
                if (at == 0) a.few_partial_ml[to] = f32x2{big, total};
            }
        }
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------
//
// A workgroup owns 128 or 256 rows of one key/value head (prompts, or the rows of many sequences behind a common prefix): the matrix
// units bound this kernel, with the vector units' exponentials and scales close by.  Keys and values go through the LDS in tiles that its four or eight
// wavefronts share, made 16 bits wide on their way, double buffered with one barrier a tile; a wavefront owns 32 rows.  Scores as [token][row] = K Q^T, results as [head_dim][row] = V^T P^T in the 32x32x16 shape; maxima and
// sums stay in a lane but for one exchange between the halves.
//
// 32 heads of 128, 8 of keys and values, 2048 tokens behind 6144: 275 us, 875 TFLOP/s, the matrix units busy 37 % and the vector units 52 % of the cycles; a
// prompt of 4096 with 32 heads of each 168 us, 820 TFLOP/s (by 128 rows 188: a tile is made wide for half the rows); heads of 64 110 us, 625 TFLOP/s.  With the
// value scale in the exponent, a multiplication less, registers spill for heads of 64 (215 us), and heads of 128 gain nothing.  Little work costs latency: a
// workgroup's first tile begins 4.5 us after the launch, and its results take 2 us.
template <int D, int WAVES> struct TileLds {
    static constexpr int kTile = D == 256 ? 32 : 64; // tokens
    uint8_t k[2][kTile * 2 * D], v[2][kTile * 2 * D];
    int32_t p[32 * WAVES];
};

template <typename T, int D, int WAVES> __device__ __forceinline__ void many_rows(const AttentionArgs &a, TileLds<D, WAVES> &lds, bool common, uint32_t block)
{
    typedef TileLds<D, WAVES> Lds;
    constexpr int kTile = Lds::kTile, KS = D / 16, DT = D / 32, HT = kTile / 32; // HT: 32-token products of a tile
    constexpr uint32_t kRows = 32 * WAVES, kRowBytes = 2 * D, kChunks = D / 16, kRowsALoad = 64 / kChunks; // rows: in the LDS; chunks: of 16 bytes in the cache
    constexpr int kTokens = kTile / WAVES, kLoads = kTokens / (int)kRowsALoad; // tokens that a wavefront brings, in so many loads
    constexpr int kKnown = 64 / WAVES; // tiles that are known at once
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
                const uint32_t rows = b + lane < a.batch.n_seqs && end_s > first_s ? min(end_s - first_s, a.max_new) * a.group : 0;
                const uint32_t tiles = rows > a.least_many ? (rows + kRows - 1) / kRows : 0;
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
        for (uint32_t i = threadIdx.x; i < kRows; i += 64 * WAVES) lds.p[i] = kNoPosition;
        __syncthreads();
        const uint32_t r_low = i_first / a.group, r_high = min((i_first + kRows - 1) / a.group + 1, a.batch.n_rows);
        for (uint32_t b = threadIdx.x; b < a.batch.n_seqs; b += 64 * WAVES) {
            const uint32_t first = a.batch.first_row(b), end = a.batch.rows_end(b);
            const int32_t len = first < end ? a.batch.length(b) : 0;
            for (uint32_t r = max(first, r_low); r < min(end, r_high); r++)
                for (uint32_t i = max(r * a.group, i_first); i < min((r + 1) * a.group, i_first + kRows); i++) lds.p[i - i_first] = len - (int32_t)(end - r);
        }
        __syncthreads();
        int32_t p_low = kNoPosition, p_high = kNoPosition;
#pragma unroll
        for (uint32_t i = 0; i < kRows; i += 64) {
            const int32_t p = lds.p[i + lane];
            p_low = p_low == kNoPosition ? p : p == kNoPosition ? p_low : min(p_low, p), p_high = max(p_high, p);
        }
        range_of_positions(p_low, p_high, p_min, p_max);
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
    f16x8 q[KS];
    f32x16 o[DT];
    float ref = 0.0f; // what the weights are relative to, in powers of two: kLiftMany or more below the largest score
    bool any = false; // a score has been seen
    float l = 0.0f;
    const T *q_src = static_cast<const T *>(a.q) + my_packed * a.q_row + my_head * a.q_head + 8 * half;
    u32x4 raw[KS];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < KS; i++) {
        raw[i] = u32x4{};
        if (my_row < n) raw[i] = *reinterpret_cast<const u32x4 *>(q_src + 16 * i);
        if (a.negate) raw[i] ^= 0x80008000u;
        most = largest(most, raw[i]);
    }
    const Queries<T> as_f16(largest_over_32(most));
    const float row_scale = fminf(fmaxf(a.scale * as_f16.back, 0x1p-149f), 0x1p127f);
#pragma unroll
    for (int i = 0; i < KS; i++) q[i] = as_f16(raw[i]);
    ValueScale value_scale;
    value_scale.begin(my_row < n);
#pragma unroll
    for (int dt = 0; dt < DT; dt++) o[dt] = f32x16{};

    const int32_t *prefix_table = a.batch.prefix_pages, *own_table = a.batch.pages + (uint64_t)seq * a.batch.pages_stride;
    const uint64_t page_stride = (uint64_t)a.n_kv_heads << a.batch.page_shift;
    const uint64_t head_at = (uint64_t)kv << a.batch.page_shift;
    const uint32_t place_mask = (1u << a.batch.page_shift) - 1u;
    // What there is to know of kKnown tiles, so many tiles ahead: lane l has, of tile i + l / WAVES counted from t_begin, where the tokens that wavefront
    // l mod WAVES brings lie in the pools (in bytes; where there is no page, those of page 0, which are then taken for hidden), and the tile's
    // flags.  A tile's step takes its own with three reads of a lane.  (Scalar loads would do for the pages, but the LDS's data are waited
    // for by the same counter, all of it.)
    enum : uint32_t {
        kThere = (1 << WAVES) - 1, // a bit for each wavefront's tokens: they are there
        kPrefix = 256,  // of the prefix's table
        kSome = 512,    // this wavefront's rows see some of it,
        kEdge = 1024    // and not all of it
    };
    struct Known {
        uint32_t low, high, flags;
        float ks, vs;
    };
    auto pages_from = [&](int32_t i) {
        const int32_t t = t_begin + i + (int32_t)(lane / WAVES), j = first_token(t) + (int32_t)(lane % WAVES) * kTokens;
        const bool in_prefix = t < prefix_tiles.count;
        int32_t e = -1;
        if (t < t_end && j < (in_prefix ? base : all_last.high)) e = in_prefix ? prefix_table[(uint32_t)j >> a.batch.page_shift] : own_table[(uint32_t)(j - base) >> a.batch.page_shift];
        return (uint32_t)e < a.batch.n_pages ? e : -1;
    };
    auto known_from = [&](int32_t i, int32_t page) {
        const int32_t t = t_begin + i + (int32_t)(lane / WAVES), j = first_token(t);
        const bool in_prefix = t < prefix_tiles.count;
        const uint32_t place = (uint32_t)(j + (int32_t)(lane % WAVES) * kTokens - (in_prefix ? 0 : base)) & place_mask;
        const uint64_t token = page_stride * (uint32_t)max(page, 0) + head_at + place, at = token * D;
        const uint32_t all_there = (uint32_t)(__ballot(page >= 0) >> (lane / WAVES * WAVES)) & kThere;
        // scales of 16 tokens that no row sees may be anything
        const int32_t j16 = j + (int32_t)(lane % WAVES * kTokens & ~15u);
        const bool is_seen = page >= 0 && j16 < min(in_prefix ? base : 0x7FFFFFFF, all_last.high) && (j16 + 16 > all_first.low || j16 < all_last.sinks);
        const bool whole = all_there == kThere && (!in_prefix || j + kTile <= base);
        const bool some = t < t_end && j < last_sees.high && (j + kTile > first_sees.low || j < last_sees.sinks);
        const bool edge = !whole || j + kTile > first_sees.high || (j < last_sees.low && j + kTile > first_sees.sinks);
        return Known{(uint32_t)at, (uint32_t)(at >> 32), all_there | (in_prefix ? kPrefix : 0u) | (some ? kSome : 0u) | (edge ? kEdge : 0u),
                     is_seen ? sound_scale(a.k_scales[token >> a.block_shift]) : 0x1p-126f, is_seen ? sound_scale(a.v_scales[token >> a.block_shift]) : 0x1p-126f};
    };
    int32_t pages_ahead = pages_from(0);
    Known known = known_from(0, pages_ahead);
    pages_ahead = pages_from(kKnown);
    auto flags_of = [&](int32_t i) { return (uint32_t)__builtin_amdgcn_readlane((int)known.flags, WAVES * (i & (kKnown - 1))); };
    // tokens from here on are not of the tile's table
    auto end_of = [&](uint32_t flags) { return flags & kPrefix ? base : 0x7FFFFFFF; };
    u32x4 k_new[kLoads], v_new[kLoads];
    const uint32_t lane_at = lane * 16;
    auto bring = [&](int32_t i) {
        const int32_t l = WAVES * (i & (kKnown - 1)) + (int32_t)wave;
        const uint64_t at = (uint32_t)__builtin_amdgcn_readlane((int)known.low, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)known.high, l) << 32;
        const uint8_t *k_at = static_cast<const uint8_t *>(a.k_pages) + at, *v_at = static_cast<const uint8_t *>(a.v_pages) + at;
#pragma unroll
        for (int i = 0; i < kLoads; i++) k_new[i] = *reinterpret_cast<const u32x4 *>(k_at + lane_at + i * 1024);
#pragma unroll
        for (int i = 0; i < kLoads; i++) v_new[i] = *reinterpret_cast<const u32x4 *>(v_at + lane_at + i * 1024);
    };
    // Keys and values lie in the LDS in 16 bits, a chunk of the cache as two of 16 bytes.  A token's chunks lie exchanged, so that 16 tokens' same chunks are on
    // different banks, the same four of 4 tokens', and every other one that 8 lanes store.
    auto place_of = [](uint32_t token, uint32_t chunk) {
        const uint32_t other = D == 64 ? (token >> 1 & 1u) << 2 | ((token >> 2 & 3u) ^ (token & 1u)) : ((token & 3u) << 2 | (token >> 2 & 3u)) ^ (chunk >> 3 & 1u);
        return token * kRowBytes + ((chunk ^ other) << 4);
    };
    const uint32_t lds_k = dcdev::lds_address(&lds) + offsetof(Lds, k), lds_v = dcdev::lds_address(&lds) + offsetof(Lds, v);
    // where a lane puts what it brings, and where it reads its part of the first operands
    uint32_t put_at[kLoads][2], k_at[KS], v_at[DT][2];
#pragma unroll
    for (int i = 0; i < kLoads; i++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t token = wave * kTokens + i * kRowsALoad + lane / kChunks, chunk = 2 * (lane % kChunks) + h;
            put_at[i][h] = place_of(token, chunk);
        }
#pragma unroll
    for (int i = 0; i < KS; i++) k_at[i] = place_of(c, 2 * i + half);
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t i16 = lane & 15u, token = 4 * half + (i16 >> 2) + 8 * h, chunk = 4 * dt + 2 * (lane >> 4 & 1u) + (i16 >> 1 & 1u);
            v_at[dt][h] = place_of(token, chunk) + (i16 & 1u) * 8;
        }
    uint32_t next_ks[2 * HT], next_vs[2 * HT];
    auto put = [&](int32_t i, uint32_t buffer) {
        // scales of its 16 tokens each, of keys and of values
#pragma unroll
        for (int u = 0; u < 2 * HT; u++) {
            const int32_t l = WAVES * (i & (kKnown - 1)) + u * (16 / kTokens);
            next_ks[u] = (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(known.ks), l);
            next_vs[u] = (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(known.vs), l);
        }
#pragma unroll
        for (int i = 0; i < kLoads; i++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                *(lds_u32x4 *)(uintptr_t)(lds_k + buffer * kBuffer + put_at[i][h]) = eight_f16(k_new[i][2 * h], k_new[i][2 * h + 1]);
                *(lds_u32x4 *)(uintptr_t)(lds_v + buffer * kBuffer + put_at[i][h]) = eight_f16(v_new[i][2 * h], v_new[i][2 * h + 1]);
            }
    };
    auto k_operand = [&](int i, uint32_t buffer) {
        return __builtin_bit_cast(f16x8, *(const lds_u32x4 *)(uintptr_t)(lds_k + buffer * kBuffer + 32 * (i / KS) * kRowBytes + k_at[i % KS]));
    };
    auto v_operand = [&](int i, uint32_t buffer) {
        const u32x2 lo = lds_column4(lds_v + buffer * kBuffer + 16 * (i / DT) * kRowBytes + v_at[i % DT][0]);
        const u32x2 hi = lds_column4(lds_v + buffer * kBuffer + 16 * (i / DT) * kRowBytes + v_at[i % DT][1]);
        return __builtin_bit_cast(f16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    };

    // A step works on tile t, whose keys and values are in buffer B, while the next tile's go from registers into the other buffer and those
    // of the tile behind it are asked for.
    uint32_t flags = 0, flags_next = 0; // of tiles t and t + 1
    auto step = [&](auto B, int32_t t) {
        constexpr uint32_t buffer = decltype(B)::value;
        constexpr int kProducts = HT * KS, kGroups = 2 * HT, kAhead = 4;
        uint32_t ks[2 * HT], vs[2 * HT];
#pragma unroll
        for (int u = 0; u < 2 * HT; u++) ks[u] = next_ks[u], vs[u] = next_vs[u];
        if (t + 1 < t_end) put(t + 1 - t_begin, buffer ^ 1u);
        const int32_t i_after = t + 2 - t_begin;
        if ((i_after & (kKnown - 1)) == 0) {
            known = known_from(i_after, pages_ahead);
            pages_ahead = pages_from(i_after + kKnown);
        }
        const uint32_t flags_after = flags_of(i_after);
        if (t + 2 < t_end) bring(i_after);

        // a wavefront whose rows see nothing of the tile has nothing to do
        if (flags & kSome) {
            f32x16 s[HT];
            float scale[2 * HT]; // of 16 tokens' scores
#pragma unroll
            for (int u = 0; u < 2 * HT; u++) scale[u] = fminf(fmaxf(__uint_as_float(ks[u]) * row_scale, 0x1p-149f), 0x1p127f);
            f16x8 x[kAhead];
            // The operands come out of the LDS several products ahead of their use.
#pragma unroll
            for (int i = 0; i < kAhead; i++) x[i] = k_operand(i, buffer);
#pragma unroll
            for (int i = 0; i < kProducts; i++) {
                s[i / KS] = Mfma<_Float16>::m32(x[i % kAhead], q[i % KS], i % KS ? s[i / KS] : f32x16{});
                if (i + kAhead < kProducts) x[i % kAhead] = k_operand(i + kAhead, buffer);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
            for (int i = 0; i < kProducts - kAhead; i++) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
            uint32_t most_vs = 0;
#pragma unroll
            for (int u = 0; u < 2 * HT; u++) most_vs = max(most_vs, vs[u]);
            uint32_t row_vs = most_vs; // of what the row sees
            if (flags & kEdge) {
                const int32_t j = first_token(t);
                Seen here = seen;
                here.high = min(here.high, end_of(flags));
                row_vs = 0;
#pragma unroll
                for (int u = 0; u < 2 * HT; u++) row_vs = max(row_vs, here.some_of16(j + 16 * u) ? vs[u] : 0u);
#pragma unroll
                for (int h = 0; h < HT; h++)
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const int token = 32 * h + 8 * (i / 4) + i % 4; // of the lower half; the upper half's is 4 further, brought by the same wavefront
                        const bool sees = here.token(j + token + 4 * (int32_t)half) & ((flags >> (token / kTokens) & 1u) != 0);
                        s[h][i] = sees ? s[h][i] : -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2 * HT; u++) {
                float most = s[u / 2][8 * (u % 2)];
#pragma unroll
                for (int i = 1; i < 7; i += 2) most = fmaxf(fmaxf(most, s[u / 2][8 * (u % 2) + i]), s[u / 2][8 * (u % 2) + i + 1]); // one operation
                top = fmaxf(top, fmaxf(most, s[u / 2][8 * (u % 2) + 7]) * scale[u]);
            }
            top = max_over_32(top);
            // The reference moves, to kLiftMany below the largest score so far, only when one is so far above it that its weight would exceed
            // 2^(kLiftMany + 8): what has been added up is scaled now and then, not for every tile.
            if (__any(top - ref > kLiftMany + 8.0f || (!any && top != -INFINITY))) {
                const float next = any ? fmaxf(ref, top - kLiftMany) : top == -INFINITY ? 0.0f : top - kLiftMany;
                const float fade = any ? exp2_of(ref - next) : 0.0f;
                any = any || top != -INFINITY;
                l *= fade;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[dt] *= fade;
                ref = next;
            }
            if (__any(value_scale.below(most_vs))) {
                const float less = value_scale.take_in(row_vs);
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[dt] *= less;
            }
            f16x8 w[kGroups], y[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; i++) y[i] = v_operand(i, buffer);
#pragma unroll
            for (int u = 0; u < kGroups; u++) {
                f32x8 e;
#pragma unroll
                for (int i = 0; i < 8; i++) e[i] = exp2_of(__builtin_fmaf(s[u / 2][8 * (u % 2) + i], scale[u], -ref));
                l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                w[u] = __builtin_convertvector(e * value_scale.share(__uint_as_float(vs[u])), f16x8);
            }
#pragma unroll
            for (int i = 0; i < kGroups * DT; i++) {
                o[i % DT] = Mfma<_Float16>::m32(y[i % kAhead], w[i / DT], o[i % DT]);
                if (i + kAhead < kGroups * DT) y[i % kAhead] = v_operand(i + kAhead, buffer);
            }
            dcdev::in_register<false>(l); // the additions among the products, not behind them
        }
        flags = flags_next, flags_next = flags_after;
        __syncthreads();
    };

    if (t_begin < t_end) {
        flags = flags_of(0), flags_next = flags_of(1);
        bring(0);
        put(0, 0);
        if (t_begin + 1 < t_end) bring(1);
    }
    __syncthreads();
    for (int32_t t = t_begin; t < t_end; t += 2) {
        step(std::integral_constant<uint32_t, 0>{}, t);
        if (t + 1 < t_end) step(std::integral_constant<uint32_t, 1>{}, t + 1);
    }

    const f32x2 both = swapped32(l);
    const float total = (both[0] + both[1]) * __uint_as_float((127u - kLiftMany) << 23);
    // what the weights are relative to (also if the row saw scores and none was a number)
    const float top = any || total != total ? ref + kLiftMany : -INFINITY;
    if (my_row >= n) return;
    uint32_t row = my_row; // where the results go is worked out here, not kept in registers from the beginning
    dcdev::anew(row);
    const uint32_t packed = row_first + row / a.group, head = kv * a.group + row % a.group;
    const float by = value_scale.value() * __uint_as_float((127u - kLiftMany) << 23);
    auto sums = [&](int dt, int b) { return f32x4{o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]} * by; };
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

template <typename T, int D, int RT> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void dc_attention_i8_few_kernel(AttentionArgs a)
{
    __shared__ __align__(16) FewLds<D, RT> lds;
    const bool common = blockIdx.x < a.prefix.blocks;
    few_rows<T, D, RT>(a, common ? a.prefix : a.own, lds, common, common ? blockIdx.x : blockIdx.x - a.prefix.blocks);
}

template <typename T, int D, int WAVES> __global__ __launch_bounds__(64 * WAVES, workgroups_a_unit<D>()) void dc_attention_i8_tile_kernel(AttentionArgs a)
{
    __shared__ __align__(16) TileLds<D, WAVES> lds;
    const bool common = blockIdx.x < a.prefix.blocks;
    many_rows<T, D, WAVES>(a, lds, common, common ? blockIdx.x : blockIdx.x - a.prefix.blocks);
}

// A common prefix with many rows and few rows in each sequence: the first is bound by the matrix units, the second by memory, and a compute unit has some of each.
// The prefix's workgroups come first.  (In turn by eights they fell on every other group of compute units, two to a unit: 64 sequences behind 16384
// tokens 62.5 us, so 48.8, 5 of them the join; 256 of them 167 and 118, 40 sequences and heads behind 4096 82 and 79, 64 of 4000 behind 16384 104 and 109.)
// A workgroup's XCD is its number modulo 8, and those of one key/value head's prefix stay on one.
template <typename T, int D, int RT> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void dc_attention_i8_both_kernel(AttentionArgs a)
{
    __shared__ __align__(16) union {
        FewLds<D, RT> few;
        TileLds<D, 4> many;
    } lds;
    if (blockIdx.x < a.prefix.blocks) many_rows<T, D, 4>(a, lds.many, true, blockIdx.x);
    else few_rows<T, D, RT>(a, a.own, lds.few, false, blockIdx.x - a.prefix.blocks);
}

// Sequences with many rows, and among them some with at most 16 (a prompt, or a piece of one, among generated tokens), which only the device can tell: these are
// taken as few rows, behind the others; two to a workgroup of 512 threads.  8 heads of 128 for 32 (us; all as many rows, and so): 2048 tokens and 63 sequences of one
// token over 4096 264 and 153 (the parts alone 74 and 85), 512 behind 1536 and 32 of them 175 and 114; where all have many rows, 852 workgroups of heads of
// 64, 67.8 and 68.9.
template <typename T, int D, int WAVES, bool APART> __global__ __launch_bounds__(64 * WAVES, workgroups_a_unit<D>()) void dc_attention_i8_mixed_kernel(AttentionArgs a)
{
    __shared__ __align__(16) union {
        FewLds<D, 1> few[WAVES / 4];
        TileLds<D, WAVES> many;
    } lds;
    const uint32_t many = a.prefix.blocks + a.own.blocks;
    if (blockIdx.x < many) {
        const bool common = blockIdx.x < a.prefix.blocks;
        many_rows<T, D, WAVES>(a, lds.many, common, common ? blockIdx.x : blockIdx.x - a.prefix.blocks);
    } else {
        const uint32_t team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), item = (blockIdx.x - many) * (WAVES / 4) + team;
        if (item < a.few.blocks) few_rows<T, D, 1, APART>(a, a.few, lds.few[team], false, item);
    }
}
template <typename T, int D, int WAVES> void launch_mixed(const AttentionArgs &a, hipStream_t stream)
{
    constexpr uint32_t kTeams = WAVES / 4;
    const dim3 grid(a.prefix.blocks + a.own.blocks + (a.few.blocks + kTeams - 1) / kTeams), threads(64 * WAVES);
    if (a.few_rows_a_seq) hipLaunchKernelGGL((dc_attention_i8_mixed_kernel<T, D, WAVES, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((dc_attention_i8_mixed_kernel<T, D, WAVES, false>), grid, threads, 0, stream, a);
}

template <typename T, int D> void launch(const AttentionArgs &a, const Plan &plan, hipStream_t stream)
{
    const dim3 threads(256);
    if (a.prefix.blocks && plan.prefix_kind == kTile && plan.own_kind != kTile) {
        const dim3 grid(a.prefix.blocks + a.own.blocks);
        if (plan.own_kind == kFew16) hipLaunchKernelGGL((dc_attention_i8_both_kernel<T, D, 1>), grid, threads, 0, stream, a);
        else if constexpr (D < 256) hipLaunchKernelGGL((dc_attention_i8_both_kernel<T, D, 2>), grid, threads, 0, stream, a);
    } else { // a sequence's rows are never more than the batch's: both parts are of the kind of their rows together, or the prefix is alone
        const Kind kind = a.prefix.blocks ? std::max(plan.prefix_kind, plan.own_kind) : plan.own_kind;
        const dim3 grid(a.prefix.blocks + a.own.blocks);
        if (kind == kFew16) hipLaunchKernelGGL((dc_attention_i8_few_kernel<T, D, 1>), grid, threads, 0, stream, a);
        else if (kind == kTile) {
            if constexpr (wide_tile_rows(D) > kTileRows) {
                if (plan.tile_rows > kTileRows) {
                    if (a.few.blocks) launch_mixed<T, D, 8>(a, stream);
                    else hipLaunchKernelGGL((dc_attention_i8_tile_kernel<T, D, 8>), grid, dim3(512), 0, stream, a);
                    return;
                }
            }
            if (a.few.blocks) launch_mixed<T, D, 4>(a, stream);
            else hipLaunchKernelGGL((dc_attention_i8_tile_kernel<T, D, 4>), grid, threads, 0, stream, a);
        }
        else if constexpr (D < 256) hipLaunchKernelGGL((dc_attention_i8_few_kernel<T, D, 2>), grid, threads, 0, stream, a);
    }
}

template <typename T> void launch_d(const AttentionArgs &a, const Plan &plan, uint32_t head_dim, hipStream_t stream)
{
    if (head_dim == 64) launch<T, 64>(a, plan, stream);
    else if (head_dim == 128) launch<T, 128>(a, plan, stream);
    else launch<T, 256>(a, plan, stream);
}

} // namespace

void dcattn::launch_i8(const AttentionArgs &a, const Plan &plan, uint32_t rows_type, uint32_t head_dim, hipStream_t stream)
{
    if (rows_type == DC_TYPE_BF16) launch_d<__bf16>(a, plan, head_dim, stream);
    else launch_d<_Float16>(a, plan, head_dim, stream);
}
