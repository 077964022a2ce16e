// Rotary positions and cache append: new tokens' queries and keys are turned by their positions, keys and values go into the
// pages of their sequences.
//
// A pair (a, b) of a head becomes (a c - b s, b c + a s) with the cosine and sine of the row's position: two multiplications and
// two fused ones for 8 to 16 bytes moved, so the call is bound by memory for many rows and by the launch for few.  A thread owns
// 16 values of a head that hold whole pairs (8 of the first half and their partners in the second, or 16 neighbours): two
// 16-byte accesses each way, no exchange between lanes, and queries may be turned in place.  Results are stored past the caches'
// keeping: 2048 fp32 rows of 96 heads of 128 take 24.0 instead of 27.0 us (6.3 TB/s), 8192 rows of 120 in 16 bits 98 instead of 101 (5.2).
// (Loads that way gain only where the rows are more than the caches hold, and lose up to a fifth below.)
#include "dc_device.h"
#include "dc_pages.h"

using namespace dcpages;

namespace {

constexpr uint32_t kThreads = 256;

struct AppendArgs {
    Batch batch;
    const void *k, *v, *q;
    void *k_pages, *v_pages, *q_out;
    const float *cos, *sin;
    const int32_t *position;
    uint64_t k_row, k_head, v_row, v_head, q_row, q_head, q_out_row, q_out_head;
    uint32_t n_heads, n_kv_heads, rot_dim, n_positions, max_new;
};

template <typename X> __device__ __forceinline__ f32x8 widened(const X *p)
{
    return __builtin_convertvector(*reinterpret_cast<const typename Vec8<X>::type *>(p), f32x8);
}
__device__ __forceinline__ f32x8 widened(const float *p) { return *reinterpret_cast<const f32x8_at16 *>(p); }

// X: type of the rows, T: type of the cache, D: head_dim, NEIGHBOURS: which values are a pair; WAVES: wavefronts that go
// through all of a row's heads; 0: a workgroup takes as many of a row's heads as it has threads for.
template <typename X, typename T, int D, bool NEIGHBOURS, int WAVES> __global__ __launch_bounds__(kThreads) void dc_kv_append_kernel(AppendArgs a)
{
    typedef typename Vec8<T>::type TV;
    constexpr uint32_t kUnits = D / 16;
    const uint32_t row = WAVES == 1 ? blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    if (WAVES == 1 && row >= a.batch.n_rows) return;
    const uint32_t seq = a.batch.sequence_of(row, a.max_new);
    if (seq >= a.batch.n_seqs) return;
    const uint32_t end = a.batch.rows_end(seq);
    // row - end >= -n_rows and length >= 0: no overflow; negative for rows of a sequence that is shorter than its rows
    const int32_t pos = a.batch.length(seq) - (int32_t)(end - row);
    const bool placed = pos >= 0 && pos < a.batch.capacity();
    const int32_t page = placed ? a.batch.page_of(seq, (uint32_t)pos) : -1;

    const uint32_t unit = threadIdx.x % kUnits;
    const bool turns = 16 * unit < a.rot_dim;
    f32x8 c = 1.0f, s = 0.0f;
    if (a.rot_dim) {
        const int32_t at = a.position ? a.position[row] : pos;
        if ((uint32_t)at >= a.n_positions) return;
        if (turns) {
            const uint64_t o = (uint64_t)(uint32_t)at * (a.rot_dim / 2) + 8 * unit;
            c = *reinterpret_cast<const f32x8_at16 *>(a.cos + o);
            s = *reinterpret_cast<const f32x8_at16 *>(a.sin + o);
        }
    }
    // where the thread's two groups of 8 values begin
    const uint32_t first = turns && !NEIGHBOURS ? 8 * unit : 16 * unit;
    const uint32_t second = turns && !NEIGHBOURS ? a.rot_dim / 2 + 8 * unit : 16 * unit + 8;

    const uint32_t slots = a.n_heads + 2 * a.n_kv_heads;
    constexpr uint32_t kStep = (WAVES == 1 ? 64 : kThreads) / kUnits;
    const uint32_t slots_begin = WAVES ? 0 : blockIdx.y * kStep, slots_end = WAVES ? slots : min(slots, slots_begin + kStep);
    const uint32_t slot_first = slots_begin + (WAVES == 1 ? threadIdx.x & 63u : threadIdx.x) / kUnits;
#pragma unroll 4
    for (uint32_t slot = slot_first; slot < slots_end; slot += kStep) {
        const bool is_q = slot < a.n_heads, is_k = !is_q && slot < a.n_heads + a.n_kv_heads;
        const uint32_t head = is_q ? slot : slot - a.n_heads - (is_k ? 0u : a.n_kv_heads);
        if (!is_q && page < 0) continue;
        const X *src = is_q ? static_cast<const X *>(a.q) + row * a.q_row + head * a.q_head
                     : is_k ? static_cast<const X *>(a.k) + row * a.k_row + head * a.k_head
                            : static_cast<const X *>(a.v) + row * a.v_row + head * a.v_head;
        const uint64_t in_pages = ((((uint64_t)(uint32_t)page * a.n_kv_heads + head) << a.batch.page_shift) +
                                   a.batch.place_in_page((uint32_t)pos)) * D;
        T *dst = is_q ? static_cast<T *>(a.q_out) + row * a.q_out_row + head * a.q_out_head
                      : (is_k ? static_cast<T *>(a.k_pages) : static_cast<T *>(a.v_pages)) + in_pages;
        f32x8 x = widened(src + first), y = widened(src + second);
        if (turns && (is_q || is_k)) {
            if (NEIGHBOURS) {
                f32x8 u, w;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    u[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
                    u[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
                    w[2 * i] = y[2 * i] * c[4 + i] - y[2 * i + 1] * s[4 + i];
                    w[2 * i + 1] = y[2 * i + 1] * c[4 + i] + y[2 * i] * s[4 + i];
                }
                x = u, y = w;
            } else {
                const f32x8 u = x * c - y * s;
                y = y * c + x * s;
                x = u;
            }
        }
        __builtin_nontemporal_store(__builtin_convertvector(x, TV), reinterpret_cast<TV *>(dst + first));
        __builtin_nontemporal_store(__builtin_convertvector(y, TV), reinterpret_cast<TV *>(dst + second));
    }
}

template <typename X, typename T, int D, int WAVES> void launch_w(const AppendArgs &a, bool neighbours, dim3 grid, hipStream_t stream)
{
    if (neighbours) hipLaunchKernelGGL((dc_kv_append_kernel<X, T, D, true, WAVES>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((dc_kv_append_kernel<X, T, D, false, WAVES>), grid, dim3(kThreads), 0, stream, a);
}

template <typename X, typename T, int D> void launch_d(const AppendArgs &a, bool neighbours, hipStream_t stream)
{
    const uint32_t slots = a.n_heads + 2 * a.n_kv_heads, slots_a_block = kThreads / (D / 16), rows = a.batch.n_rows;
    // Few rows: a row's heads are asked for all at once (128 to 512 rows: 3.1 to 4.1 instead of 4.1 to 4.7 us; 2048 rows of 48 heads 10.5 instead
    // of 10.1).  Many: the cosines and sines stay in registers for all of a row's heads, of which a workgroup takes a row, or if they are not
    // enough for its threads four (rows of 2 x 5 to 20 heads of 64: 4.0 instead of 5.3 us for 3000, 5.1 instead of 6.3 for 3500; 8192 rows of 48
    // heads of 128: 33 instead of 31.4).
    if (rows < 512) {
        const dim3 grid(rows, (slots + slots_a_block - 1) / slots_a_block);
        launch_w<X, T, D, 0>(a, neighbours, grid, stream);
    } else if (slots < slots_a_block) {
        launch_w<X, T, D, 1>(a, neighbours, dim3((rows + 3) / 4), stream);
    } else {
        launch_w<X, T, D, 4>(a, neighbours, dim3(rows), stream);
    }
}

template <typename X, typename T> void launch(const AppendArgs &a, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (head_dim == 64) launch_d<X, T, 64>(a, neighbours, stream);
    else if (head_dim == 128) launch_d<X, T, 128>(a, neighbours, stream);
    else launch_d<X, T, 256>(a, neighbours, stream);
}

template <typename T> void launch_x(const AppendArgs &a, uint32_t type, uint32_t head_dim, bool neighbours, hipStream_t stream)
{
    if (type == DC_TYPE_BF16) launch<__bf16, T>(a, head_dim, neighbours, stream);
    else if (type == DC_TYPE_F16) launch<_Float16, T>(a, head_dim, neighbours, stream);
    else launch<float, T>(a, head_dim, neighbours, stream);
}

} // namespace

extern "C" int dc_kv_append(const dc_kv_cache *cache, const dc_kv_batch *batch, const dc_kv_rows *rows, void *hip_stream)
{
    if (!cache_ok(cache) || !batch_ok(cache, batch) || !rows) return DC_E_ARG;
    const uint32_t d = cache->head_dim;
    if (rows->type > DC_TYPE_F32 || rows->n_heads > 65535 || rows->pairing > DC_ROPE_NEIGHBOURS || rows->rot_dim % 16 || rows->rot_dim > d)
        return DC_E_ARG;
    if (!rows->k_dev || !rows->v_dev || !aligned16(rows->k_dev) || !aligned16(rows->v_dev) ||
        !strides_ok(rows->k_row_stride, rows->k_head_stride) || !strides_ok(rows->v_row_stride, rows->v_head_stride))
        return DC_E_ARG;
    if (rows->n_heads) {
        if (!rows->q_dev || !rows->q_out_dev || !aligned16(rows->q_dev) || !aligned16(rows->q_out_dev) ||
            !strides_ok(rows->q_row_stride, rows->q_head_stride) ||
            !strides_apart(rows->q_out_row_stride, rows->q_out_head_stride, batch->n_rows, rows->n_heads, d))
            return DC_E_ARG;
        if (rows->q_dev == rows->q_out_dev && (rows->type != cache->type || rows->q_row_stride != rows->q_out_row_stride ||
                                               rows->q_head_stride != rows->q_out_head_stride))
            return DC_E_ARG;
    }
    if (rows->rot_dim && (!rows->cos_dev || !rows->sin_dev || !aligned16(rows->cos_dev) || !aligned16(rows->sin_dev) || rows->n_positions < 1))
        return DC_E_ARG;

    AppendArgs a = {};
    a.batch = batch_args(cache, batch);
    a.k = rows->k_dev, a.v = rows->v_dev, a.q = rows->q_dev;
    a.k_pages = cache->k_dev, a.v_pages = cache->v_dev, a.q_out = rows->q_out_dev;
    a.cos = rows->cos_dev, a.sin = rows->sin_dev, a.position = rows->position_dev;
    a.k_row = rows->k_row_stride, a.k_head = rows->k_head_stride, a.v_row = rows->v_row_stride, a.v_head = rows->v_head_stride;
    a.q_row = rows->q_row_stride, a.q_head = rows->q_head_stride;
    a.q_out_row = rows->q_out_row_stride, a.q_out_head = rows->q_out_head_stride;
    a.n_heads = rows->n_heads, a.n_kv_heads = cache->n_kv_heads, a.rot_dim = rows->rot_dim, a.n_positions = rows->n_positions;
    a.max_new = batch->max_new;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool neighbours = rows->pairing == DC_ROPE_NEIGHBOURS;
    if (cache->type == DC_TYPE_BF16) launch_x<__bf16>(a, rows->type, d, neighbours, stream);
    else launch_x<_Float16>(a, rows->type, d, neighbours, stream);
    return dc_launch_status();
}
