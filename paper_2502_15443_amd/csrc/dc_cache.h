// What the kernels of the cache append share, whatever the cache's type.
#ifndef DC_CACHE_H
#define DC_CACHE_H

#include "dc_device.h"
#include "dc_pages.h"

namespace dccache {

using namespace dcpages;

constexpr uint32_t kThreads = 256;

struct AppendArgs {
    Batch batch;
    const void *k, *v, *q;
    void *k_pages, *v_pages, *q_out;
    const float *cos, *sin;
    const int32_t *position;
    uint64_t k_row, k_head, v_row, v_head, q_row, q_head, q_out_row, q_out_head;
    uint32_t n_heads, n_kv_heads, rot_dim, n_positions, max_new;
    // of a cache of 8 bits: scale of [page][head][token >> block_shift]; turned queries are f16, else bf16
    float *k_scales, *v_scales;
    uint32_t block_shift;
    bool rows_f16;
};

template <typename X> __device__ __forceinline__ f32x8 widened(const X *p)
{
    return __builtin_convertvector(*reinterpret_cast<const typename Vec8<X>::type *>(p), f32x8);
}
__device__ __forceinline__ f32x8 widened(const float *p) { return *reinterpret_cast<const f32x8_at16 *>(p); }

// The append to a cache of 8 bits.
void launch_i8(const AppendArgs &a, uint32_t x_type, uint32_t head_dim, bool neighbours, hipStream_t stream);

} // namespace dccache

#endif // DC_CACHE_H
