// Rotary positions and append to a cache of 8 bits: queries and keys are turned by their positions, keys and values are held as whole numbers
// with a scale for each block of tokens of a head.
//
// A block's scale is the smallest power of two s >= 2^-126 with |x| <= 127 s for its values; a value is held as the whole number nearest to
// x / s, which for a power of two is x times its reciprocal, exactly (for a scale that somebody else wrote and that is none, see nearest).  A block that the call's rows do not reach back to the beginning of has
// earlier tokens: its scale only grows, and then their numbers are rounded to the larger steps.  So the call must see all of a block's new rows
// together: the row that is the first of its block in this call takes care of the block (its leader).
#include "dc_cache.h"

#include <math.h>

#include <algorithm>

using namespace dccache;

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A leader with at most this many rows takes care of its block beside the row's queries; one with more has threads for its block.
constexpr uint32_t kFewRows = 4, kMostThreads = 1024;

// Where a row belongs, and the block that it leads, if it is a leader.  Its page is looked at last: the row's values need not wait for it.
struct Place {
    uint32_t count; // rows of the block, from this one on; 0 for a row that leads none
    int32_t pos, entry;
    uint32_t in_page;
    __device__ __forceinline__ Place(const AppendArgs &a, uint32_t row, uint32_t seq, uint32_t first, uint32_t end, int32_t length) : count(0), entry(-1), in_page(0)
    {
        // row - end >= -n_rows and length >= 0: no overflow; negative for rows of a sequence that is shorter than its rows
        pos = length - (int32_t)(end - row);
        if (pos < 0 || pos >= a.batch.capacity()) return;
        entry = a.batch.page_of(seq, (uint32_t)pos);
        in_page = a.batch.place_in_page((uint32_t)pos);
        const uint32_t block = 1u << a.block_shift, in_block = in_page & (block - 1u);
        if (in_block && row != first) return;
        count = min(block - in_block, first + min(end - first, a.max_new) - row);
        if ((uint32_t)pos < a.batch.prefix_len) count = min(count, a.batch.prefix_len - (uint32_t)pos);
    }
};

// Smallest power of two s >= 2^-126 with most <= 127 s; 127 = (1 + 0x7E0000 2^-23) 2^6.
__device__ __forceinline__ float scale_for(float most)
{
    const uint32_t u = __float_as_uint(most);
    return __uint_as_float((uint32_t)max(1, (int32_t)(u >> 23) - 6 + ((u & 0x7FFFFFu) > 0x7E0000u)) << 23);
}
// 1 / s, for a power of two without a division.
__device__ __forceinline__ float reciprocal(float s)
{
    const uint32_t u = __float_as_uint(s);
    return u & 0x7FFFFFu || u > 253u << 23 ? 1.0f / s : __uint_as_float((254u << 23) - u);
}

// A thread's 16 values of a head, in two groups of 8 that hold whole pairs.
struct Values {
    f32x8 x, y;
};

template <typename T> __device__ __forceinline__ dcdev::u32x4 rounded(const f32x8 &x)
{
    return __builtin_bit_cast(dcdev::u32x4, __builtin_convertvector(x, typename Vec8<T>::type));
}

// The same as they lie in memory.
template <typename X> struct Raw {
    typename Vec8<X>::type x, y;
    __device__ __forceinline__ void load(const X *p, const X *q) { x = *reinterpret_cast<const typename Vec8<X>::type *>(p), y = *reinterpret_cast<const typename Vec8<X>::type *>(q); }
    __device__ __forceinline__ Values values() const { return Values{__builtin_convertvector(x, f32x8), __builtin_convertvector(y, f32x8)}; }
};
template <> struct Raw<float> {
    f32x8 x, y;
    __device__ __forceinline__ void load(const float *p, const float *q) { x = widened(p), y = widened(q); }
    __device__ __forceinline__ Values values() const { return Values{x, y}; }
};

// Which values those are; what does not turn is taken as it lies.
template <bool NEIGHBOURS> struct Unit {
    bool turns;
    uint32_t first, second;
    __device__ __forceinline__ Unit(const AppendArgs &a, uint32_t unit)
        : turns(16 * unit < a.rot_dim), first(turns && !NEIGHBOURS ? 8 * unit : 16 * unit),
          second(turns && !NEIGHBOURS ? a.rot_dim / 2 + 8 * unit : 16 * unit + 8) {}
};

struct Angles {
    f32x8 c, s;
    bool given; // false: the row's cosines lie outside the table
};
__device__ __forceinline__ Angles angles_of(const AppendArgs &a, uint32_t row, int32_t pos, uint32_t unit, bool turns)
{
    Angles t{1.0f, 0.0f, true};
    if (!a.rot_dim) return t;
    const int32_t at = a.position ? a.position[row] : pos;
    t.given = (uint32_t)at < a.n_positions;
    if (turns && t.given) {
        const uint64_t o = (uint64_t)(uint32_t)at * (a.rot_dim / 2) + 8 * unit;
        t.c = *reinterpret_cast<const f32x8_at16 *>(a.cos + o);
        t.s = *reinterpret_cast<const f32x8_at16 *>(a.sin + o);
    }
    return t;
}

// Every product and sum is rounded: what is held in 8 bits is the same whoever turns it.
template <bool NEIGHBOURS> __device__ __forceinline__ Values turned(const Values &v, const Angles &t)
{
#pragma clang fp contract(off)
    Values r;
    if (NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            r.x[2 * i] = v.x[2 * i] * t.c[i] - v.x[2 * i + 1] * t.s[i];
            r.x[2 * i + 1] = v.x[2 * i + 1] * t.c[i] + v.x[2 * i] * t.s[i];
            r.y[2 * i] = v.y[2 * i] * t.c[4 + i] - v.y[2 * i + 1] * t.s[4 + i];
            r.y[2 * i + 1] = v.y[2 * i + 1] * t.c[4 + i] + v.y[2 * i] * t.s[4 + i];
        }
    } else {
        r.x = v.x * t.c - v.y * t.s;
        r.y = v.y * t.c + v.x * t.s;
    }
    return r;
}

// Largest magnitude of the values, and whether all are numbers.  (A sum of magnitudes is no number if one of them is none; if it only leaves the range,
// the values are looked at one by one for nothing.)
struct Most {
    float value;
    bool numbers;
    __device__ __forceinline__ explicit Most(const Values &v) : value(0.0f)
    {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) value = fmaxf(fmaxf(value, fabsf(v.x[i])), fabsf(v.y[i])), sum += fabsf(v.x[i]) + fabsf(v.y[i]);
        numbers = sum < INFINITY;
        if (!numbers) {
            dcdev::keep_order(); // a branch, not selections: it is hardly ever taken
            value = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = fabsf(v.x[i]), y = fabsf(v.y[i]);
                value = fmaxf(value, fmaxf(x < INFINITY ? x : 0.0f, y < INFINITY ? y : 0.0f));
            }
        }
    }
};

__device__ __forceinline__ bool power_of_two(float s) { return (__float_as_uint(s) & 0x7FFFFFu) == 0; }
// The whole number nearest to x / s, ties to even: rint(x / s) with a quotient that may be off in its last bits, or one of that number's neighbours.  Which side of
// the middle between two x lies on comes out of one rounding, which leaves the sign and zero as they are: what small scales take below the normal range is
// lifted by 2^64 before.
__device__ __forceinline__ int32_t nearest(float x, float s, float quotient)
{
    const float lift = s < 1.0f ? 0x1p64f : 1.0f, n = rintf(quotient);
    x *= lift, s *= lift;
    const float above = __builtin_fmaf(-(n + 0.5f), s, x), below = __builtin_fmaf(-(n - 0.5f), s, x);
    const int32_t i = (int32_t)n;
    return i + (above > 0.0f || (above == 0.0f && (i & 1))) - (below < 0.0f || (below == 0.0f && (i & 1)));
}

// The whole numbers nearest to 8 values / scale, as bytes, of which `by` is the reciprocal.  A power of two's is exact; added to 1.5 2^23, a number of up to 127 is
// rounded to the nearest whole one, ties to even, and its low byte is what is wanted.  Infinities are 127 with their sign, NaN is 0.
// plain: the values are numbers, and the scale a power of two.
__device__ __forceinline__ u32x2 whole_numbers(const f32x8 &x, float scale, float by, bool plain)
{
#pragma clang fp contract(off)
    u32x2 w;
    if (plain) {
        uint32_t n[8];
#pragma unroll
        for (int i = 0; i < 8; i++) n[i] = __float_as_uint(x[i] * by + 12582912.0f);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t low = __builtin_amdgcn_perm(n[4 * h + 1], n[4 * h], 0x0C0C0400u), high = __builtin_amdgcn_perm(n[4 * h + 3], n[4 * h + 2], 0x0C0C0400u);
            w[h] = __builtin_amdgcn_perm(high, low, 0x05040100u);
        }
    } else { // hardly ever: short rather than fast
        f32x8 left = x;
        uint64_t bytes = 0;
#pragma unroll 1
        for (int i = 0; i < 8; i++) {
            const uint32_t u = __float_as_uint(left[0]), most = u >> 31 ? (uint32_t)-127 : 127u;
            const uint32_t n = (u & 0x7FFFFFFFu) < 0x7F800000u ? (uint32_t)nearest(left[0], scale, left[0] * by) : u & 0x7FFFFFu ? 0u : most;
            bytes = bytes >> 8 | (uint64_t)n << 56;
            left = __builtin_shufflevector(left, left, 1, 2, 3, 4, 5, 6, 7, 0);
        }
        w = u32x2{(uint32_t)bytes, (uint32_t)(bytes >> 32)};
    }
    return w;
}
// 16 bytes' whole numbers of a scale `before`, of a larger one that is a power of two and has the reciprocal `by`.
__device__ __forceinline__ dcdev::u32x4 in_larger_steps(const dcdev::u32x4 &from, float before, float by)
{
    dcdev::u32x4 to;
    const float less = before * by;
    if (power_of_two(before)) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
            to[k] = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) to[k] |= ((uint32_t)(int32_t)rintf((float)(int8_t)(from[k] >> (8 * i)) * less) & 255u) << (8 * i);
        }
    } else { // (the product of a number and such a scale can be rounded to the middle between two)
        dcdev::u32x4 left = from;
        to = dcdev::u32x4{};
#pragma unroll 1
        for (int k = 0; k < 16; k++) {
            const float q = (float)(int8_t)left[0], n = rintf(q * less);
            const float above = __builtin_fmaf(q, less, -(n + 0.5f)), below = __builtin_fmaf(q, less, -(n - 0.5f));
            const int32_t whole = (int32_t)n, i = whole + (above > 0.0f || (above == 0.0f && (whole & 1))) - (below < 0.0f || (below == 0.0f && (whole & 1)));
            // all 16 bytes by one: out at the low end, in at the high end
            const dcdev::u32x4 next_left = {left[1], left[2], left[3], 0u}, next_to = {to[1], to[2], to[3], (uint32_t)i};
#pragma unroll
            for (int j = 0; j < 4; j++) {
                left[j] = (uint32_t)(((uint64_t)next_left[j] << 32 | left[j]) >> 8);
                to[j] = (uint32_t)(((uint64_t)next_to[j] << 32 | to[j]) >> 8);
            }
        }
    }
    return to;
}

// A row's queries (QUERIES), and blocks with few new rows (KEYS).  A thread owns 16 values of a head of the row, D / 16 neighbouring ones a head.
template <typename X, int D, bool NEIGHBOURS, bool QUERIES, bool KEYS> __device__ __forceinline__ void append_row(const AppendArgs &a, uint32_t row, uint32_t slot_first, uint32_t slots_end, uint32_t step)
{
    constexpr uint32_t kUnits = D / 16;
    const uint32_t seq = a.batch.sequence_of(row, a.max_new);
    if (seq >= a.batch.n_seqs) return;
    const Place p(a, row, seq, a.batch.first_row(seq), a.batch.rows_end(seq), a.batch.length(seq));
    const uint32_t unit = threadIdx.x % kUnits;
    const Unit<NEIGHBOURS> u(a, unit);
    const Angles mine = angles_of(a, row, p.pos, unit, u.turns);
    const uint32_t block = 1u << a.block_shift, in_block = p.in_page & (block - 1u);
    uint32_t slot = slot_first;
    if (QUERIES && mine.given) {
#pragma unroll 4
        for (; slot < min(slots_end, a.n_heads); slot += step) {
            const uint32_t head = slot;
            const X *src = static_cast<const X *>(a.q) + row * a.q_row + head * a.q_head;
            uint16_t *dst = static_cast<uint16_t *>(a.q_out) + row * a.q_out_row + head * a.q_out_head;
            Values v{widened(src + u.first), widened(src + u.second)};
            if (u.turns) v = turned<NEIGHBOURS>(v, mine);
            dcdev::u32x4 x, y;
            if (a.rows_f16) x = rounded<_Float16>(v.x), y = rounded<_Float16>(v.y);
            else x = rounded<__bf16>(v.x), y = rounded<__bf16>(v.y);
            __builtin_nontemporal_store(x, reinterpret_cast<dcdev::u32x4 *>(dst + u.first));
            __builtin_nontemporal_store(y, reinterpret_cast<dcdev::u32x4 *>(dst + u.second));
        }
    }
    if (!KEYS || p.count == 0 || p.count > kFewRows) return;
    for (slot = slot_first; slot < slots_end; slot += step) {
        if (slot < a.n_heads) continue;
        const bool is_k = slot < a.n_heads + a.n_kv_heads;
        const uint32_t head = slot - a.n_heads - (is_k ? 0u : a.n_kv_heads);
        const uint64_t row_stride = is_k ? a.k_row : a.v_row;
        const X *src = (is_k ? static_cast<const X *>(a.k) + head * a.k_head : static_cast<const X *>(a.v) + head * a.v_head) + row * row_stride;
        auto values = [&](uint32_t i, bool &given) {
            const Angles t = i ? angles_of(a, row + i, p.pos + (int32_t)i, unit, u.turns) : mine;
            given = t.given;
            Values v{widened(src + i * row_stride + u.first), widened(src + i * row_stride + u.second)};
            return is_k && u.turns ? turned<NEIGHBOURS>(v, t) : v;
        };
        bool given;
        Values v = values(0, given);
        const uint64_t head_at = (uint64_t)(uint32_t)max(p.entry, 0) * a.n_kv_heads + head;
        float *scale_at = (is_k ? a.k_scales : a.v_scales) + (head_at << (a.batch.page_shift - a.block_shift)) + (p.in_page >> a.block_shift);
        const float before = in_block ? sound_scale(*scale_at) : 0.0f;
        const Most m(v);
        float most = given ? m.value : 0.0f;
        bool any = given, numbers = m.numbers;
#pragma unroll 1
        for (uint32_t i = 1; i < p.count; i++) {
            bool g;
            const Values w = values(i, g);
            if (!g) continue;
            const Most m(w);
            most = fmaxf(most, m.value), any = true, numbers &= m.numbers;
        }
#pragma unroll
        for (uint32_t k = 1; k < kUnits; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
        if (!any || p.entry < 0) continue;
        uint8_t *dst = static_cast<uint8_t *>(is_k ? a.k_pages : a.v_pages) + ((head_at << a.batch.page_shift) + p.in_page) * D;
        const float scale = fmaxf(scale_for(most), before), by = reciprocal(scale);
        const bool plain = numbers & power_of_two(scale);
#pragma unroll 1
        for (uint32_t i = 0; i < p.count; i++) {
            if (i) v = values(i, given);
            if (!given) continue;
            *reinterpret_cast<u32x2 *>(dst + i * D + u.first) = whole_numbers(v.x, scale, by, plain);
            *reinterpret_cast<u32x2 *>(dst + i * D + u.second) = whole_numbers(v.y, scale, by, plain);
        }
        if (in_block && scale != before) {
            uint8_t *at = dst - in_block * D + 16 * unit;
#pragma unroll 2
            for (uint32_t i = 0; i < in_block; i++) {
                dcdev::u32x4 *e = reinterpret_cast<dcdev::u32x4 *>(at + i * D);
                *e = in_larger_steps(*e, before, by);
            }
        }
        if (unit == 0) *scale_at = scale;
    }
}

// The blocks led by a row among `block` neighbouring ones that have more than `few` new rows, of some heads of the keys or of the values, one after the
// other.  A team of threads has a head's block, each of them 16 values of ROWS rows, whose cosines and sines it keeps for all heads.
// Small blocks (up to 2048 values) are a wavefront's: no barrier; else the team is the workgroup, of 256 to 1024 threads, and the next head's values
// are on their way while this head's maximum is found.  8192 rows of 40 heads of 128 in blocks of 64: 59 us for 252 MB, 4.3 TB/s, the vector units busy 46 % (14
// operations a value); 1280 workgroups of 512 threads meet 512 places, which hold what is under way at once, and neither two heads ahead (no change) nor two blocks a team (212 registers, 167 us) gives more.
// BIG: a block has more than 16 values for each of 1024 threads; those of its further rows are read twice.
template <typename X, int D, bool NEIGHBOURS, int ROWS, bool BIG> __device__ __forceinline__ void append_blocks(const AppendArgs &a, uint32_t few, uint32_t group, bool is_k, uint32_t head_first,
                                                                                                                uint32_t heads, uint32_t (&lds_most)[2][kMostThreads / 64])
{
    constexpr bool kWave = ROWS > 0; // ROWS 0: the workgroup, a row to a thread
    constexpr int kRows = kWave ? ROWS : 1;
    constexpr uint32_t kUnits = D / 16;
    const uint32_t block = 1u << a.block_shift, lane = threadIdx.x & 63u;
    const uint32_t t = kWave ? lane : threadIdx.x, tokens = (kWave ? 64u : blockDim.x) / kUnits; // rows at a time
    const uint32_t unit = t % kUnits, token = t / kUnits;
    const Unit<NEIGHBOURS> u(a, unit);
    const bool turns = is_k && u.turns, all_turn = is_k && a.rot_dim == D;
    const uint64_t row_stride = is_k ? a.k_row : a.v_row, head_stride = is_k ? a.k_head : a.v_head;
    const X *rows = static_cast<const X *>(is_k ? a.k : a.v);
    float *scales = is_k ? a.k_scales : a.v_scales;
    uint8_t *pages = static_cast<uint8_t *>(is_k ? a.k_pages : a.v_pages);

    for (uint32_t r = group * block; r < min((group + 1) * block, a.batch.n_rows); r += 64) {
        // a lane to a row: its sequence, by halving
        const uint32_t my_row = r + lane;
        uint32_t low = 0, high = a.batch.n_seqs; // the last sequence that begins at or before the row, and as rows follow one another the only one that has it
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if (a.batch.first_row(mid) <= my_row) low = mid;
            else high = mid;
        }
        const uint32_t first_row = a.batch.first_row(low), rows_end = a.batch.rows_end(low);
        const int32_t length = a.batch.length(low);
        const bool has = lane < block && my_row < a.batch.n_rows && first_row <= my_row && my_row < rows_end && my_row - first_row < a.max_new;
        // (a row that no sequence has is as if at a position below zero)
        const Place p(a, has ? my_row : 0, low, has ? first_row : 0, has ? rows_end : 1, has ? length : 0);
        uint64_t leaders = __ballot(p.count > few);
        while (leaders) {
            const int l = __builtin_ctzll(leaders);
            leaders &= leaders - 1;
            const uint32_t row = r + (uint32_t)l, count = (uint32_t)__builtin_amdgcn_readlane((int)p.count, l);
            const uint32_t in_page = (uint32_t)__builtin_amdgcn_readlane((int)p.in_page, l), in_block = in_page & (block - 1u);
            const int32_t pos = __builtin_amdgcn_readlane(p.pos, l);
            const uint32_t heads_end = head_first + heads;
            Angles angles[kRows];
            bool given[kRows];
#pragma unroll
            for (int i = 0; i < kRows; i++) {
                const uint32_t n = min(token + i * tokens, count - 1);
                angles[i] = angles_of(a, row + n, pos + (int32_t)n, unit, turns);
                given[i] = token + i * tokens < count && angles[i].given;
            }
            const X *first = rows + (row + token) * row_stride;
            Raw<X> next[kRows] = {};
            auto load = [&](uint32_t head) {
                const X *src = first + head * head_stride;
#pragma unroll
                for (int i = 0; i < kRows; i++)
                    if (given[i]) next[i].load(src + i * tokens * row_stride + u.first, src + i * tokens * row_stride + u.second);
            };
            load(head_first);
            const int32_t entry = __builtin_amdgcn_readlane(p.entry, l);
            if (entry < 0) continue;
            const uint64_t page = (uint32_t)entry;
            auto scale_at = [&](uint32_t head) {
                return scales + (((page * a.n_kv_heads + head) << (a.batch.page_shift - a.block_shift)) + (in_page >> a.block_shift));
            };
            // of the rows that a thread comes to behind its first one
            auto further = [&](const X *src, auto use) {
                if constexpr (BIG) {
#pragma unroll 1
                    for (uint32_t n = token + tokens; n < count; n += tokens) {
                        const Angles w = angles_of(a, row + n, pos + (int32_t)n, unit, turns);
                        if (!w.given) continue;
                        const X *at = src + (n - token) * row_stride;
                        const Values x{widened(at + u.first), widened(at + u.second)};
                        use(n, turns ? turned<NEIGHBOURS>(x, w) : x);
                    }
                }
            };
            uint32_t buffer = 0;
#pragma unroll 1
            for (uint32_t head = head_first; head < heads_end; head++, buffer ^= 1u) {
                const X *src = first + head * head_stride;
                const float before = in_block ? sound_scale(*scale_at(head)) : 0.0f;
                Values v[kRows];
                uint32_t most = 0; // bits of the largest magnitude and 1 more; 0: there are no values
                bool numbers = true;
                auto look = [&](const Values &v) {
                    const Most m(v);
                    most = max(most, __float_as_uint(m.value) + 1u), numbers &= m.numbers;
                };
#pragma unroll
                for (int i = 0; i < kRows; i++) {
                    v[i] = next[i].values();
                    if (all_turn) {
                        v[i] = turned<NEIGHBOURS>(v[i], angles[i]);
                    } else if (turns) {
                        dcdev::keep_order();
                        v[i] = turned<NEIGHBOURS>(v[i], angles[i]);
                    }
                }
                if (head + 1 < heads_end) load(head + 1);
#pragma unroll
                for (int i = 0; i < kRows; i++)
                    if (given[i]) look(v[i]);
                further(src, [&](uint32_t, const Values &x) { look(x); });
                most = largest_of_lanes(most);
                if constexpr (!kWave) {
                    if (lane == 0) lds_most[buffer][threadIdx.x >> 6] = most;
                    __syncthreads();
                    const uint32_t of_wave = lds_most[buffer][lane & 15u];
                    most = largest_of_lanes((lane & 15u) < blockDim.x / 64 ? of_wave : 0u);
                }
                if (!most) continue;
                const float scale = fmaxf(scale_for(__uint_as_float(most - 1u)), before), by = reciprocal(scale);
                const bool plain = numbers & power_of_two(scale);
                uint8_t *dst = pages + (((page * a.n_kv_heads + head) << a.batch.page_shift) + in_page) * D;
                auto store = [&](uint32_t n, const Values &x) {
                    *reinterpret_cast<u32x2 *>(dst + n * D + u.first) = whole_numbers(x.x, scale, by, plain);
                    *reinterpret_cast<u32x2 *>(dst + n * D + u.second) = whole_numbers(x.y, scale, by, plain);
                };
#pragma unroll
                for (int i = 0; i < kRows; i++)
                    if (given[i]) store(token + i * tokens, v[i]);
                further(src, store);
                if (in_block && scale != before) {
#pragma unroll 1
                    for (uint32_t i = token; i < in_block; i += tokens) {
                        dcdev::u32x4 *e = reinterpret_cast<dcdev::u32x4 *>(dst - (in_block - i) * D + 16 * unit);
                        *e = in_larger_steps(*e, before, by);
                    }
                }
                if (t == 0) *scale_at(head) = scale;
            }
            if constexpr (!kWave) __syncthreads(); // the next leader begins with the first buffer again
        }
    }
}

// Blocks: items are `block` neighbouring rows for each of head_groups groups of `heads` heads of keys and of values by turns; those of the same rows go to
// one XCD (a workgroup's is its number modulo 8), for they read the same cosines.
struct BlockWork {
    uint64_t items;
    uint32_t head_groups, heads, few;
};
template <typename X, int D, bool NEIGHBOURS, int ROWS, bool BIG> __device__ __forceinline__ void block_item(const AppendArgs &a, const BlockWork &w, uint64_t item,
                                                                                                             uint32_t (&most)[2][kMostThreads / 64])
{
    constexpr uint32_t kTeams = ROWS ? kThreads / 64 : 1;
    const uint32_t wave = ROWS ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const uint32_t eight = (uint32_t)(item >> 3) * kTeams + wave; // of eight groups of rows
    const uint32_t part = eight % (2 * w.head_groups), head = part / 2 * w.heads;
    append_blocks<X, D, NEIGHBOURS, ROWS, BIG>(a, w.few, eight / (2 * w.head_groups) * 8 + (uint32_t)(item & 7u), part % 2 == 0, head, min(w.heads, a.n_kv_heads - head), most);
}

// Rows: each in `parts` parts of part_slots heads (queries, then keys, then values, from number first_slot on), which row_threads threads go through.
struct RowWork {
    uint64_t items;
    uint32_t first_slot, slots_end, parts, part_slots, row_threads;
};
template <typename X, int D, bool NEIGHBOURS, bool QUERIES, bool KEYS> __device__ __forceinline__ void row_item(const AppendArgs &a, const RowWork &w, uint64_t item)
{
    const uint32_t team = __builtin_amdgcn_readfirstlane(threadIdx.x / w.row_threads), thread = threadIdx.x % w.row_threads;
    const uint64_t i = item * (blockDim.x / w.row_threads) + team, row = i / w.parts;
    const uint32_t begin = w.first_slot + (uint32_t)(i % w.parts) * w.part_slots;
    if (row < a.batch.n_rows)
        append_row<X, D, NEIGHBOURS, QUERIES, KEYS>(a, (uint32_t)row, begin + thread / (D / 16), min(w.slots_end, begin + w.part_slots), w.row_threads / (D / 16));
}

template <typename X, int D, bool NEIGHBOURS, int ROWS, bool BIG> __global__ __launch_bounds__(ROWS ? kThreads : kMostThreads) void dc_kv_append_i8_blocks_kernel(AppendArgs a, BlockWork w)
{
    __shared__ uint32_t most[2][kMostThreads / 64];
    for (uint64_t item = blockIdx.x; item < w.items; item += gridDim.x) block_item<X, D, NEIGHBOURS, ROWS, BIG>(a, w, item, most);
}
template <typename X, int D, bool NEIGHBOURS, bool QUERIES, bool KEYS> __global__ __launch_bounds__(kThreads) void dc_kv_append_i8_rows_kernel(AppendArgs a, RowWork w)
{
    for (uint64_t item = blockIdx.x; item < w.items; item += gridDim.x) row_item<X, D, NEIGHBOURS, QUERIES, KEYS>(a, w, item);
}
// Both in one launch, where there is little to do.
template <typename X, int D, bool NEIGHBOURS, int ROWS> __global__ __launch_bounds__(ROWS ? kThreads : kMostThreads) void dc_kv_append_i8_both_kernel(AppendArgs a, BlockWork b, RowWork r)
{
    __shared__ uint32_t most[2][kMostThreads / 64];
    if (blockIdx.x < b.items) block_item<X, D, NEIGHBOURS, ROWS, false>(a, b, blockIdx.x, most);
    else row_item<X, D, NEIGHBOURS, true, true>(a, r, blockIdx.x - b.items);
}

constexpr uint64_t kMostItems = 1u << 21; // of a grid; what is beyond is the same workgroups' too

// Rows' heads from number `first` to `end` on.
template <int D> RowWork row_work(uint32_t rows, uint32_t first, uint32_t end, uint32_t row_threads, uint32_t threads)
{
    const uint32_t step = row_threads / (D / 16), slots = end - first, teams = threads / row_threads;
    RowWork r = {};
    r.first_slot = first, r.slots_end = end, r.row_threads = row_threads;
    r.parts = rows < 512 ? (slots + step - 1) / step : 1;
    r.part_slots = r.parts > 1 ? step : slots;
    r.items = ((uint64_t)rows * r.parts + teams - 1) / teams;
    return r;
}
template <typename X, int D, bool NEIGHBOURS, bool QUERIES, bool KEYS> void launch_rows(const AppendArgs &a, const RowWork &r, hipStream_t stream)
{
    hipLaunchKernelGGL((dc_kv_append_i8_rows_kernel<X, D, NEIGHBOURS, QUERIES, KEYS>), dim3((uint32_t)std::min(r.items, kMostItems)), dim3(kThreads), 0, stream, a, r);
}

template <typename X, int D, bool NEIGHBOURS, int ROWS, bool BIG> void launch_n(const AppendArgs &a, const BlockWork &b, uint32_t threads, hipStream_t stream)
{
    const uint32_t rows = a.batch.n_rows, slots = a.n_heads + 2 * a.n_kv_heads;
    // One launch is shorter than several (264 rows of 32/8 heads: 5.1 and 10.0 us); with several each part has its own number of registers and threads.
    if constexpr (!BIG) {
        const RowWork r = row_work<D>(rows, 0, slots, kThreads, threads);
        if (rows < 512 && b.items + r.items <= kMostItems) {
            hipLaunchKernelGGL((dc_kv_append_i8_both_kernel<X, D, NEIGHBOURS, ROWS>), dim3((uint32_t)(b.items + r.items)), dim3(threads), 0, stream, a, b, r);
            return;
        }
    }
    const uint32_t row_threads = rows >= 512 && slots * (D / 16) <= 128 ? 64 : kThreads;
    // A sequence has at most two blocks with few rows, its first and its last one: beside many blocks they are the same kernel's (8192 rows of 40/40 heads of
    // 128 94 us, with a launch for them 101; 2048 rows of 32/8 14.2 and 16.4).  Queries have a launch of their own, 36 us for 168 MB of 40 heads (256 threads
    // have 32 heads at a time: of the second time three quarters are idle); mixed with the blocks' in one, 2048 rows take 13.3 us, but 8192 104.
    BlockWork all = b;
    if ((uint64_t)a.batch.n_seqs * 16 <= rows >> a.block_shift) all.few = 0;
    hipLaunchKernelGGL((dc_kv_append_i8_blocks_kernel<X, D, NEIGHBOURS, ROWS, BIG>), dim3((uint32_t)std::min(b.items, kMostItems)), dim3(threads), 0, stream, a, all);
    if (all.few == 0) {
        launch_rows<X, D, NEIGHBOURS, true, false>(a, row_work<D>(rows, 0, a.n_heads, row_threads, kThreads), stream);
    // Else queries apart from the blocks with few rows, which take twice the registers, if they are worth a launch (8192 rows of 40/40 heads of 128: 101
    // instead of 107 us; 2048 rows of 32/8 17.6 instead of 16.1, 32768 rows of 16/2 of 64 58 instead of 47).
    } else if (rows >= 4096 && a.n_heads * D >= 4096) {
        launch_rows<X, D, NEIGHBOURS, false, true>(a, row_work<D>(rows, a.n_heads, slots, 64, kThreads), stream);
        launch_rows<X, D, NEIGHBOURS, true, false>(a, row_work<D>(rows, 0, a.n_heads, kThreads, kThreads), stream);
    } else {
        launch_rows<X, D, NEIGHBOURS, true, true>(a, row_work<D>(rows, 0, slots, row_threads, kThreads), stream);
    }
}

template <typename X, int D, bool NEIGHBOURS> void launch_d(const AppendArgs &a, hipStream_t stream)
{
    const uint32_t block = 1u << a.block_shift, rows = a.batch.n_rows, slots = a.n_heads + 2 * a.n_kv_heads;
    if (a.max_new <= kFewRows) { // no block has more
        launch_rows<X, D, NEIGHBOURS, true, true>(a, row_work<D>(rows, 0, slots, rows >= 512 && slots * (D / 16) <= 128 ? 64 : kThreads, kThreads), stream);
        return;
    }
    const bool small = block * D <= 2048;
    const uint32_t threads = small ? kThreads : std::min(D / 16 * block, kMostThreads), teams = small ? kThreads / 64 : 1;
    const uint64_t groups = (rows + block - 1) / block;
    BlockWork b = {};
    b.few = kFewRows;
    b.heads = 1;
    while (b.heads < a.n_kv_heads && b.heads < 8 && groups * 2 * ((a.n_kv_heads + b.heads - 1) / b.heads) * (small ? 64 : threads) > 2048 * kThreads) b.heads++;
    b.head_groups = (a.n_kv_heads + b.heads - 1) / b.heads;
    b.items = ((groups + 7) / 8 * 2 * b.head_groups + teams - 1) / teams * 8;
    if (!small && D / 16 * block > kMostThreads) launch_n<X, D, NEIGHBOURS, 0, true>(a, b, threads, stream);
    else if (!small) launch_n<X, D, NEIGHBOURS, 0, false>(a, b, threads, stream);
    else if constexpr (D < 256) {
        if (D == 128 || block == 32) launch_n<X, D, NEIGHBOURS, 2, false>(a, b, threads, stream);
        else if constexpr (D == 64) launch_n<X, D, NEIGHBOURS, 1, false>(a, b, threads, stream);
    }
}

template <typename X, int D> void launch_p(const AppendArgs &a, bool neighbours, hipStream_t stream)
{
    if (neighbours) launch_d<X, D, true>(a, stream);
    else launch_d<X, D, false>(a, stream);
}

template <typename X> void launch(const AppendArgs &a, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (head_dim == 64) launch_p<X, 64>(a, neighbours, stream);
    else if (head_dim == 128) launch_p<X, 128>(a, neighbours, stream);
    else launch_p<X, 256>(a, neighbours, stream);
}

} // namespace

void dccache::launch_i8(const AppendArgs &a, uint32_t x_type, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (x_type == DC_TYPE_BF16) launch<__bf16>(a, head_dim, neighbours, stream);
    else if (x_type == DC_TYPE_F16) launch<_Float16>(a, head_dim, neighbours, stream);
    else launch<float>(a, head_dim, neighbours, stream);
}
