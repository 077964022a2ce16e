// What the kernels over a paged cache of keys and values share: the batch as they see it, where a row and a token are, and the
// host's checks of both descriptions.
#ifndef DC_PAGES_H
#define DC_PAGES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dc.h"

namespace dcpages {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef f32x8 f32x8_at16 __attribute__((aligned(16))); // in memory: addresses are multiples of 16 bytes, not of the vector's 32
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <typename T> struct Vec8;
template <> struct Vec8<__bf16> { typedef bf16x8 type; };
template <> struct Vec8<_Float16> { typedef f16x8 type; };

// The batch as kernels take it.  Whatever the device arrays hold, first_row / rows_end lie in [0, n_rows], a length is not negative (callers
// look up no position at or beyond the capacity) and a page that is used lies in [0, n_pages).
struct Batch {
    const int32_t *len, *pages, *row_start, *prefix_pages;
    uint32_t n_seqs, n_rows, pages_stride, prefix_len, n_pages, page_shift;

    __device__ __forceinline__ uint32_t clamped_row(int32_t r) const { return r < 0 ? 0u : min((uint32_t)r, n_rows); }
    __device__ __forceinline__ uint32_t first_row(uint32_t seq) const { return row_start ? clamped_row(row_start[seq]) : seq; }
    __device__ __forceinline__ uint32_t rows_end(uint32_t seq) const { return row_start ? clamped_row(row_start[seq + 1]) : seq + 1; }
    __device__ __forceinline__ int32_t length(uint32_t seq) const { return max(len[seq], 0); }
    // positions that a table can hold
    __device__ __forceinline__ int32_t capacity() const { return (int32_t)(prefix_len + (pages_stride << page_shift)); }
    // Page of a position inside the capacity, or -1 where there is none.
    __device__ __forceinline__ int32_t page_of(uint32_t seq, uint32_t pos) const
    {
        const int32_t p = pos < prefix_len ? prefix_pages[pos >> page_shift]
                                           : pages[(uint64_t)seq * pages_stride + ((pos - prefix_len) >> page_shift)];
        return (uint32_t)p < n_pages ? p : -1;
    }
    __device__ __forceinline__ uint32_t place_in_page(uint32_t pos) const
    {
        return (pos < prefix_len ? pos : pos - prefix_len) & ((1u << page_shift) - 1u);
    }
    // The first sequence that has a row among its first max_new ones (the same row in all lanes of the wavefront, which are all active);
    // n_seqs if there is none.
    __device__ __forceinline__ uint32_t sequence_of(uint32_t row, uint32_t max_new) const
    {
        if (!row_start) return row;
        for (uint32_t b = 0; b < n_seqs; b += 64) {
            const uint32_t i = b + (threadIdx.x & 63u);
            // (a row before the sequence's first is as if very far behind it)
            const uint64_t has = __ballot(i < n_seqs && row - clamped_row(row_start[i]) < max_new && clamped_row(row_start[i + 1]) > row);
            if (has) return b + (uint32_t)__builtin_ctzll(has);
        }
        return n_seqs;
    }
};

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

inline bool cache_ok(const dc_kv_cache *c)
{
    return c && (c->type == DC_TYPE_BF16 || c->type == DC_TYPE_F16) && c->n_kv_heads >= 1 && c->n_kv_heads <= 65535 &&
           (c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256) && c->page_tokens >= 16 && c->page_tokens <= 256 &&
           (c->page_tokens & (c->page_tokens - 1)) == 0 && c->n_pages >= 1 && c->n_pages <= 0x7FFFFFFFu && c->k_dev && c->v_dev &&
           aligned16(c->k_dev) && aligned16(c->v_dev);
}

inline bool batch_ok(const dc_kv_cache *c, const dc_kv_batch *b)
{
    if (!b || b->n_seqs < 1 || b->n_seqs > 65535 || b->n_rows < 1 || b->n_rows >= 1u << 24 || b->max_new < 1 ||
        b->max_new > b->n_rows || b->max_len < 1 || b->pages_stride < 1 || !b->len_dev || !b->pages_dev)
        return false;
    if (!b->row_start_dev && (b->n_rows != b->n_seqs || b->max_new != 1)) return false;
    if ((b->prefix_len != 0) != (b->prefix_pages_dev != nullptr)) return false;
    // kernels reckon with positions some tiles beyond the last one, in 32 bits
    return (uint64_t)b->prefix_len + (uint64_t)b->pages_stride * c->page_tokens <= 0x7FFF0000ull;
}

// A row stride and a head stride of rows that are read; of rows that are written, which must not lie over one another.
inline bool strides_ok(uint64_t row, uint64_t head) { return row % 8 == 0 && head % 8 == 0; }
inline bool strides_apart(uint64_t row, uint64_t head, uint32_t n_rows, uint32_t n_heads, uint32_t head_dim)
{
    if (!strides_ok(row, head)) return false;
    const uint64_t rows_span = (n_rows - 1ull) * row + head_dim, heads_span = (n_heads - 1ull) * head + head_dim;
    return (n_heads == 1 || head >= head_dim) && (n_rows == 1 || row >= head_dim) &&
           (n_rows == 1 || n_heads == 1 || row >= heads_span || head >= rows_span);
}

inline uint32_t shift_of(uint32_t power_of_two)
{
    uint32_t s = 0;
    while ((1u << s) < power_of_two) s++;
    return s;
}

inline Batch batch_args(const dc_kv_cache *c, const dc_kv_batch *b)
{
    return Batch{b->len_dev, b->pages_dev, b->row_start_dev, b->prefix_pages_dev, b->n_seqs, b->n_rows, b->pages_stride,
                 b->prefix_len, c->n_pages, shift_of(c->page_tokens)};
}

} // namespace dcpages

#endif // DC_PAGES_H
