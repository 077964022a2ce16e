// Rotary positions and append to a cache of 8 bits: queries and keys are turned by their positions, keys and values are held as whole numbers
// with a scale for each block of tokens of a head.
//
// A block's scale is the smallest power of two s >= 2^-126 with |x| <= 127 s for its values; a value is held as the whole number nearest to
// x / s, which for a power of two is x times its reciprocal, exactly.  A block that the call's rows do not reach back to the beginning of has
// earlier tokens: its scale only grows, and then their numbers are rounded to the larger steps.  So the call must see all of a block's new rows
// together: the row that is the first of its block in this call takes care of the block (its leader).
#include "dc_cache.h"

#include <math.h>

#include <algorithm>

using namespace dccache;

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A leader with at most this many rows takes care of its block beside the row's queries; one with more has a workgroup's threads for its block.
constexpr uint32_t kFewRows = 4;

// Where a row belongs, and the block that it leads, if it is a leader.
struct Place {
    uint32_t seq, count; // count: rows of the block, from this one on; 0 for a row that leads none, or whose page is not there
    int32_t pos, page;
    uint32_t in_page;
    __device__ __forceinline__ Place(const AppendArgs &a, uint32_t row, uint32_t seq) : seq(seq), count(0), pos(-1), page(-1), in_page(0)
    {
        if (seq >= a.batch.n_seqs) return;
        const uint32_t first = a.batch.first_row(seq), end = a.batch.rows_end(seq);
        // row - end >= -n_rows and length >= 0: no overflow; negative for rows of a sequence that is shorter than its rows
        pos = a.batch.length(seq) - (int32_t)(end - row);
        if (pos < 0 || pos >= a.batch.capacity()) return;
        page = a.batch.page_of(seq, (uint32_t)pos);
        in_page = a.batch.place_in_page((uint32_t)pos);
        const uint32_t block = 1u << a.block_shift, in_block = in_page & (block - 1u);
        if (page < 0 || (in_block && row != first)) return;
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
// A scale that is read: a number above 0.
__device__ __forceinline__ float sound_scale(float s) { return fminf(fmaxf(s, 0x1p-126f), 0x1p127f); }

// A thread's 16 values of a head, in two groups of 8 that hold whole pairs.
struct Values {
    f32x8 x, y;
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

// Largest magnitude of the values that are numbers.
__device__ __forceinline__ float largest_number(const Values &v)
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float a = fabsf(v.x[i]), b = fabsf(v.y[i]);
        m = fmaxf(m, fmaxf(a < INFINITY ? a : 0.0f, b < INFINITY ? b : 0.0f));
    }
    return m;
}

// The whole numbers nearest to 8 values times `by`, as bytes; NaN is 0.
__device__ __forceinline__ u32x2 whole_numbers(const f32x8 &x, float by)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        w[h] = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float r = rintf(x[4 * h + i] * by);
            const int32_t n = r == r ? (int32_t)fminf(fmaxf(r, -127.0f), 127.0f) : 0;
            w[h] |= ((uint32_t)n & 255u) << (8 * i);
        }
    }
    return u32x2{w[0], w[1]};
}
// 16 bytes' whole numbers times `by`, rounded.
__device__ __forceinline__ dcdev::u32x4 in_larger_steps(const dcdev::u32x4 &from, float by)
{
    dcdev::u32x4 to;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        to[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) to[k] |= ((uint32_t)(int32_t)rintf((float)(int8_t)(from[k] >> (8 * i)) * by) & 255u) << (8 * i);
    }
    return to;
}

// A row's queries, and blocks with few new rows.  A thread owns 16 values of a head of the row, D / 16 neighbouring ones a head.
template <typename X, typename T, int D, bool NEIGHBOURS> __device__ __forceinline__ void append_row(const AppendArgs &a, uint32_t row, uint32_t slot_first, uint32_t slots_end,
                                                                                                 uint32_t step)
{
    typedef typename Vec8<T>::type TV;
    constexpr uint32_t kUnits = D / 16;
    const uint32_t seq = a.batch.sequence_of(row, a.max_new);
    if (seq >= a.batch.n_seqs) return;
    const Place p(a, row, seq);
    const uint32_t unit = threadIdx.x % kUnits;
    const Unit<NEIGHBOURS> u(a, unit);
    const Angles mine = angles_of(a, row, p.pos, unit, u.turns);
    const uint32_t block = 1u << a.block_shift, in_block = p.in_page & (block - 1u);
    for (uint32_t slot = slot_first; slot < slots_end; slot += step) {
        const bool is_q = slot < a.n_heads, is_k = !is_q && slot < a.n_heads + a.n_kv_heads;
        const uint32_t head = is_q ? slot : slot - a.n_heads - (is_k ? 0u : a.n_kv_heads);
        if (is_q) {
            if (!mine.given) continue;
            const X *src = static_cast<const X *>(a.q) + row * a.q_row + head * a.q_head;
            T *dst = static_cast<T *>(a.q_out) + row * a.q_out_row + head * a.q_out_head;
            Values v{widened(src + u.first), widened(src + u.second)};
            if (u.turns) v = turned<NEIGHBOURS>(v, mine);
            __builtin_nontemporal_store(__builtin_convertvector(v.x, TV), reinterpret_cast<TV *>(dst + u.first));
            __builtin_nontemporal_store(__builtin_convertvector(v.y, TV), reinterpret_cast<TV *>(dst + u.second));
            continue;
        }
        if (p.count == 0 || p.count > kFewRows) continue;
        const uint64_t row_stride = is_k ? a.k_row : a.v_row;
        const X *src = (is_k ? static_cast<const X *>(a.k) + head * a.k_head : static_cast<const X *>(a.v) + head * a.v_head) + row * row_stride;
        const uint64_t head_at = (uint64_t)(uint32_t)p.page * a.n_kv_heads + head;
        float *scale_at = (is_k ? a.k_scales : a.v_scales) + (head_at << (a.batch.page_shift - a.block_shift)) + (p.in_page >> a.block_shift);
        uint8_t *dst = static_cast<uint8_t *>(is_k ? a.k_pages : a.v_pages) + ((head_at << a.batch.page_shift) + p.in_page) * D;
        const float before = in_block ? sound_scale(*scale_at) : 0.0f;
        auto values = [&](uint32_t i, bool &given) {
            const Angles t = i ? angles_of(a, row + i, p.pos + (int32_t)i, unit, u.turns) : mine;
            given = t.given;
            Values v{widened(src + i * row_stride + u.first), widened(src + i * row_stride + u.second)};
            return is_k && u.turns ? turned<NEIGHBOURS>(v, t) : v;
        };
        bool given;
        Values v = values(0, given);
        float most = given ? largest_number(v) : 0.0f;
        bool any = given;
        for (uint32_t i = 1; i < p.count; i++) {
            bool g;
            const Values w = values(i, g);
            if (g) most = fmaxf(most, largest_number(w)), any = true;
        }
#pragma unroll
        for (uint32_t k = 1; k < kUnits; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
        if (!any) continue;
        const float scale = fmaxf(scale_for(most), before), by = 1.0f / scale;
        for (uint32_t i = 0; i < p.count; i++) {
            if (i) v = values(i, given);
            if (!given) continue;
            *reinterpret_cast<u32x2 *>(dst + i * D + u.first) = whole_numbers(v.x, by);
            *reinterpret_cast<u32x2 *>(dst + i * D + u.second) = whole_numbers(v.y, by);
        }
        if (in_block && scale != before) {
            const float less = before * by;
            uint8_t *at = dst - in_block * D + 16 * unit;
#pragma unroll 4
            for (uint32_t i = 0; i < in_block; i++) {
                dcdev::u32x4 *e = reinterpret_cast<dcdev::u32x4 *>(at + i * D);
                *e = in_larger_steps(*e, less);
            }
        }
        if (unit == 0) *scale_at = scale;
    }
}

// The blocks led by a row among `block` neighbouring ones that have more than a few new rows, for as many heads of keys or values as a workgroup
// has threads for: a thread has 16 values of every so many of a block's rows.
template <typename X, int D, bool NEIGHBOURS> __device__ __forceinline__ void append_blocks(const AppendArgs &a, uint32_t group, uint32_t slot_group, float *lds_most)
{
    constexpr uint32_t kUnits = D / 16;
    const uint32_t block = 1u << a.block_shift, lane = threadIdx.x & 63u;
    const uint32_t slot_threads = min(kThreads, kUnits * block), tokens = slot_threads / kUnits; // of a head; of those, rows at a time
    const uint32_t slot = slot_group * (kThreads / slot_threads) + threadIdx.x / slot_threads;
    const bool is = slot < 2 * a.n_kv_heads, is_k = slot < a.n_kv_heads;
    const uint32_t head = is_k ? slot : slot - a.n_kv_heads;
    const uint32_t t = threadIdx.x % slot_threads, unit = t % kUnits, token = t / kUnits;
    const Unit<NEIGHBOURS> u(a, unit);
    const uint64_t row_stride = is_k ? a.k_row : a.v_row;
    const X *heads = is_k ? static_cast<const X *>(a.k) + head * a.k_head : static_cast<const X *>(a.v) + head * a.v_head;

    for (uint32_t r = group * block; r < min((group + 1) * block, a.batch.n_rows); r += 64) {
        // a lane to a row: its sequence, by halving
        const uint32_t my_row = r + lane;
        const bool mine = lane < block && my_row < a.batch.n_rows;
        uint32_t low = 0, high = a.batch.n_seqs; // the last sequence that begins at or before the row, and as rows follow one another the only one that has it
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if (a.batch.first_row(mid) <= my_row) low = mid;
            else high = mid;
        }
        const bool has = mine && a.batch.first_row(low) <= my_row && my_row < a.batch.rows_end(low) && my_row - a.batch.first_row(low) < a.max_new;
        const Place p(a, has ? my_row : 0, has ? low : a.batch.n_seqs);
        uint64_t leaders = __ballot(p.count > kFewRows);
        while (leaders) {
            const int l = __builtin_ctzll(leaders);
            leaders &= leaders - 1;
            const uint32_t row = r + (uint32_t)l, count = (uint32_t)__builtin_amdgcn_readlane((int)p.count, l);
            const uint32_t in_page = (uint32_t)__builtin_amdgcn_readlane((int)p.in_page, l), in_block = in_page & (block - 1u);
            const int32_t pos = __builtin_amdgcn_readlane(p.pos, l);
            const uint64_t head_at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(p.page, l) * a.n_kv_heads + head;
            float *scale_at = (is_k ? a.k_scales : a.v_scales) + (head_at << (a.batch.page_shift - a.block_shift)) + (in_page >> a.block_shift);
            uint8_t *dst = static_cast<uint8_t *>(is_k ? a.k_pages : a.v_pages) + ((head_at << a.batch.page_shift) + in_page) * D;
            const float before = is && in_block ? sound_scale(*scale_at) : 0.0f;
            auto values = [&](uint32_t i, bool &given) {
                const Angles t = angles_of(a, row + i, pos + (int32_t)i, unit, u.turns);
                given = t.given;
                const X *src = heads + (row + i) * row_stride;
                Values v{widened(src + u.first), widened(src + u.second)};
                return is_k && u.turns ? turned<NEIGHBOURS>(v, t) : v;
            };
            float most = -1.0f; // none
            if (is)
                for (uint32_t i = token; i < count; i += tokens) {
                    bool given;
                    const Values v = values(i, given);
                    if (given) most = fmaxf(most, largest_number(v));
                }
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
            if (lane == 0) lds_most[threadIdx.x >> 6] = most;
            __syncthreads();
            for (uint32_t w = 0; w < slot_threads / 64; w++) most = fmaxf(most, lds_most[(threadIdx.x / slot_threads) * (slot_threads / 64) + w]);
            __syncthreads();
            if (!is || most < 0.0f) continue;
            const float scale = fmaxf(scale_for(most), before), by = 1.0f / scale;
            for (uint32_t i = token; i < count; i += tokens) {
                bool given;
                const Values v = values(i, given);
                if (!given) continue;
                *reinterpret_cast<u32x2 *>(dst + i * D + u.first) = whole_numbers(v.x, by);
                *reinterpret_cast<u32x2 *>(dst + i * D + u.second) = whole_numbers(v.y, by);
            }
            if (in_block && scale != before) {
                const float less = before * by;
                for (uint32_t i = token; i < in_block; i += tokens) {
                    dcdev::u32x4 *e = reinterpret_cast<dcdev::u32x4 *>(dst - (in_block - i) * D + 16 * unit);
                    *e = in_larger_steps(*e, less);
                }
            }
            if (t == 0) *scale_at = scale;
        }
    }
}

// A launch's items: rows, each in row_parts parts of part_slots heads (queries, then keys, then values); and `block` neighbouring rows for each
// of slot_groups groups of heads.
struct Work {
    uint64_t row_items, block_items;
    uint32_t row_parts, part_slots, slot_groups;
};

template <typename X, typename T, int D, bool NEIGHBOURS> __global__ __launch_bounds__(kThreads) void dc_kv_append_i8_kernel(AppendArgs a, Work w)
{
    __shared__ float most[kThreads / 64];
    constexpr uint32_t kStep = kThreads / (D / 16);
    for (uint64_t item = blockIdx.x; item < w.row_items + w.block_items; item += gridDim.x) {
        if (item < w.row_items) {
            const uint32_t row = (uint32_t)(item / w.row_parts), begin = (uint32_t)(item % w.row_parts) * w.part_slots;
            append_row<X, T, D, NEIGHBOURS>(a, row, begin + threadIdx.x / (D / 16), min(a.n_heads + 2 * a.n_kv_heads, begin + w.part_slots), kStep);
        } else {
            append_blocks<X, D, NEIGHBOURS>(a, (uint32_t)((item - w.row_items) / w.slot_groups), (uint32_t)((item - w.row_items) % w.slot_groups), most);
        }
    }
}

template <typename X, typename T, int D> void launch_d(const AppendArgs &a, bool neighbours, hipStream_t stream)
{
    const uint32_t block = 1u << a.block_shift, rows = a.batch.n_rows, slots = a.n_heads + 2 * a.n_kv_heads, step = kThreads / (D / 16);
    Work w = {};
    w.row_parts = rows < 512 ? (slots + step - 1) / step : 1;
    w.part_slots = w.row_parts > 1 ? step : slots;
    w.row_items = (uint64_t)rows * w.row_parts;
    const uint32_t slot_threads = std::min<uint32_t>(kThreads, D / 16 * block), a_group = kThreads / slot_threads;
    w.slot_groups = (2 * a.n_kv_heads + a_group - 1) / a_group;
    if (a.max_new > kFewRows) w.block_items = (uint64_t)((rows + block - 1) / block) * w.slot_groups;
    const dim3 grid((uint32_t)std::min<uint64_t>(w.row_items + w.block_items, 1u << 23)); // what is beyond is the same workgroups' too
    if (neighbours) hipLaunchKernelGGL((dc_kv_append_i8_kernel<X, T, D, true>), grid, dim3(kThreads), 0, stream, a, w);
    else hipLaunchKernelGGL((dc_kv_append_i8_kernel<X, T, D, false>), grid, dim3(kThreads), 0, stream, a, w);
}

template <typename X, typename T> void launch(const AppendArgs &a, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (head_dim == 64) launch_d<X, T, 64>(a, neighbours, stream);
    else if (head_dim == 128) launch_d<X, T, 128>(a, neighbours, stream);
    else launch_d<X, T, 256>(a, neighbours, stream);
}

template <typename X> void launch_t(const AppendArgs &a, uint32_t rows_type, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (rows_type == DC_TYPE_BF16) launch<X, __bf16>(a, head_dim, neighbours, stream);
    else launch<X, _Float16>(a, head_dim, neighbours, stream);
}

} // namespace

void dccache::launch_i8(const AppendArgs &a, uint32_t x_type, uint32_t rows_type, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (x_type == DC_TYPE_BF16) launch_t<__bf16>(a, rows_type, head_dim, neighbours, stream);
    else if (x_type == DC_TYPE_F16) launch_t<_Float16>(a, rows_type, head_dim, neighbours, stream);
    else launch_t<float>(a, rows_type, head_dim, neighbours, stream);
}
