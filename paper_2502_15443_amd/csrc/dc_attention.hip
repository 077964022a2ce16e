// Attention of new tokens over a paged cache of keys and values: causal, with an optional sliding window whose first tokens stay
// visible, over private pages and a prefix that all sequences share.
//
// For a row with query q: s_j = scale (q . k_j), out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) with the running maximum m: one
// pass over the keys and values, in which a larger maximum scales what has been added up so far.
//
// A workgroup owns one row of one query head; its four wavefronts take every fourth key.  A lane holds head_dim / 64 values of the
// query, the key and the result.
#include "dc_device.h"
#include "dc_pages.h"

#include <math.h>

using namespace dcpages;

namespace {

struct AttentionArgs {
    Batch batch;
    const void *k_pages, *v_pages, *q;
    void *out;
    float *lse;
    uint64_t q_row, q_head, out_row, out_head;
    uint32_t n_heads, n_kv_heads, group, window, sinks;
    float scale;
};

__device__ __forceinline__ float sum_of_lanes(float v)
{
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) v += __shfl_xor(v, i);
    return v;
}

template <typename T, int D> __global__ __launch_bounds__(256) void dc_attention_rows_kernel(AttentionArgs a)
{
    constexpr int E = D / 64;
    const uint32_t row = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t seq = a.batch.sequence_of(row);
    if (seq >= a.batch.n_seqs) return;
    const uint32_t end = a.batch.rows_end(seq);
    const int32_t p = a.batch.length(seq) - (int32_t)(end - row), last = min(p, a.batch.capacity() - 1);
    const T *q = static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head + lane * E;
    const uint32_t kv = head / a.group;
    float qf[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < E; i++) qf[i] = (float)q[i] * a.scale, o[i] = 0.0f;
    for (int32_t j = wave; j <= last; j += 4) {
        if (a.window && (int64_t)j <= (int64_t)p - a.window && (uint32_t)j >= a.sinks) continue;
        const int32_t page = a.batch.page_of(seq, j);
        if (page < 0) continue;
        const uint64_t at = ((((uint64_t)page * a.n_kv_heads + kv) << a.batch.page_shift) + a.batch.place_in_page(j)) * D + lane * E;
        const T *k = static_cast<const T *>(a.k_pages) + at, *v = static_cast<const T *>(a.v_pages) + at;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < E; i++) s += qf[i] * (float)k[i];
        s = sum_of_lanes(s);
        if (s == -INFINITY) continue;
        const float top = fmaxf(m, s), e = expf(s - top), f = expf(m - top);
        l = l * f + e;
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = o[i] * f + e * (float)v[i];
        m = top;
    }
    __shared__ float ms[4], ls[4], os[4][D];
    if (lane == 0) ms[wave] = m, ls[wave] = l;
#pragma unroll
    for (int i = 0; i < E; i++) os[wave][lane * E + i] = o[i];
    __syncthreads();
    if (wave) return;
    float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])), sum = 0.0f, r[E] = {};
    for (int w = 0; w < 4; w++) {
        if (ls[w] == 0.0f) continue;
        const float f = expf(ms[w] - top);
        sum += ls[w] * f;
#pragma unroll
        for (int i = 0; i < E; i++) r[i] += os[w][lane * E + i] * f;
    }
    T *out = static_cast<T *>(a.out) + row * a.out_row + head * a.out_head + lane * E;
#pragma unroll
    for (int i = 0; i < E; i++) out[i] = (T)(sum == 0.0f ? 0.0f : r[i] / sum);
    if (a.lse && lane == 0) a.lse[(uint64_t)row * a.n_heads + head] = sum == 0.0f ? -INFINITY : top + logf(sum);
}

bool attention_ok(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *t)
{
    if (!cache_ok(cache) || !batch_ok(cache, batch) || !t) return false;
    if (t->n_heads < 1 || t->n_heads > 65535 || t->n_heads % cache->n_kv_heads || !isfinite(t->scale)) return false;
    return t->q_dev && t->out_dev && t->q_dev != t->out_dev && aligned16(t->q_dev) && aligned16(t->out_dev) && ((uintptr_t)t->lse_dev & 3u) == 0 &&
           strides_ok(t->q_row_stride, t->q_head_stride) &&
           strides_apart(t->out_row_stride, t->out_head_stride, batch->n_rows, t->n_heads, cache->head_dim);
}

template <typename T> void launch(const AttentionArgs &a, uint32_t head_dim, hipStream_t stream)
{
    const dim3 grid(a.batch.n_rows, a.n_heads);
    if (head_dim == 64) hipLaunchKernelGGL((dc_attention_rows_kernel<T, 64>), grid, dim3(256), 0, stream, a);
    else if (head_dim == 128) hipLaunchKernelGGL((dc_attention_rows_kernel<T, 128>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((dc_attention_rows_kernel<T, 256>), grid, dim3(256), 0, stream, a);
}

} // namespace

extern "C" int dc_attention_paged_workspace(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_attention *attention,
                                            uint64_t *workspace_bytes)
{
    if (!workspace_bytes || !attention_ok(cache, batch, attention)) return DC_E_ARG;
    *workspace_bytes = 0;
    return DC_OK;
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
    a.window = attention->window, a.sinks = attention->sinks, a.scale = attention->scale;
    if (cache->type == DC_TYPE_BF16) launch<__bf16>(a, cache->head_dim, static_cast<hipStream_t>(hip_stream));
    else launch<_Float16>(a, cache->head_dim, static_cast<hipStream_t>(hip_stream));
    return dc_launch_status();
}
