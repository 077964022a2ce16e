// What the kernels of the attention over a paged cache share, whatever the cache's type: their arguments, which tokens a row sees, exchanges
// between lanes, and where results go.
#ifndef DC_ATTENTION_H
#define DC_ATTENTION_H

#include "dc_device.h"
#include "dc_pages.h"

#include <math.h>
#include <stddef.h>

#include <type_traits>

namespace dcattn {

using namespace dcpages;

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
    Part prefix, own, few;  // few: of sequences with at most least_many rows among others with many
    uint32_t least_many;
    // The splits of those are theirs alone (0: they are as many as the others'): [sequence][row, few_rows_a_seq of them][head][slot], as above.
    uint32_t few_rows_a_seq;
    float *few_partial;
    f32x2 *few_partial_ml;
    // of a cache of 8 bits: scale of [page][head][token >> block_shift]
    const float *k_scales, *v_scales;
    uint32_t block_shift;
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
    // one of 16 tokens from j on (there may be none between low and high)
    __device__ __forceinline__ bool some_of16(int32_t j) const { return (max(low, j) < min(high, j + 16)) | (j < min(sinks, high)); }
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

constexpr uint32_t kTileRows = 128; // of a workgroup of the kernel for many rows

// Which kernel works through a part: that for at most 16 rows or 32 rows, or that for many.
enum Kind { kFew16 = 0, kFew32 = 1, kTile = 2 };
struct Plan {
    Kind prefix_kind, own_kind;
    uint32_t tile_rows; // of a workgroup of the kernel for many rows
    uint64_t few_at;    // where the workspace has what the splits of few rows among many leave
};
// Over a cache of 8 bits a workgroup has up to this many rows (of heads of 64 and 256 a half less: a wavefront's part of a tile is no whole load, or registers
// are for four wavefronts only).
constexpr uint32_t wide_tile_rows(uint32_t head_dim) { return head_dim == 128 ? 2 * kTileRows : kTileRows; }

// Tokens of a tile of the kernel for few rows over a cache of 8 bits: 64, or with 32 rows, which leave fewer registers, 32.
constexpr int few_tile(int row_tiles) { return row_tiles == 1 ? 64 : 32; }

// The kernels over a cache of 8 bits; joining, where results are in parts, is the caller's.
void launch_i8(const AttentionArgs &a, const Plan &plan, uint32_t rows_type, uint32_t head_dim, hipStream_t stream);

} // namespace dcattn

#endif // DC_ATTENTION_H
