// A step's tables from the tokens that sequences hold and get: lengths, first rows, pages taken and given back, and each row's place.
//
// Pages are taken and given back in the order of sequences and entries, so an entry's place in the queue is the number of entries before it that
// take (give back) a page: counts, their prefix sums, and the entries once more.  A wavefront works on a run of neighbouring entries of one
// sequence; few runs are one workgroup's, many a launch's for each of the three parts.
#include "dc_device.h"
#include "dc_pages.h"

#include <algorithm>

using namespace dcpages;

namespace {

constexpr uint32_t kLoads = 16, kRun = 64 * kLoads; // entries of a run
constexpr uint32_t kScanThreads = 1024;
constexpr int32_t kMostLength = 0x7FFFFFFF;

// What is known of a sequence before its entries are looked at.
struct Sequence {
    int32_t held, end; // tokens held, and with all the new ones (2^31 - 1 if they are more)
    uint32_t first_row, rows;
};
struct Queue {
    uint32_t first, count;
};
// Entries of a run that take a page, and that give one back; behind the sums, of all runs before it.
struct Moves {
    uint32_t taken, back;
};

struct TablesArgs {
    const int32_t *held, *arriving, *pages_in, *prefix_pages, *queue_in;
    int32_t *free, *len, *row_start, *pages, *queue, *position, *seq;
    int64_t *slot;
    Queue *ws_queue;
    Sequence *ws_seqs;
    Moves *ws_moves;
    uint32_t n_seqs, n_rows, page_shift, stride, n_pages, prefix_len, window, sinks;
    uint32_t runs, n_items; // runs of a sequence, of all
};

// Tokens that a sequence holds, those that it gets, and those that it has with them.
__device__ __forceinline__ uint32_t tokens_of(const TablesArgs &a, uint32_t seq, int32_t &held, int32_t &end)
{
    const int32_t n = a.arriving[seq];
    held = n < 0 ? 0 : max(a.held[seq], 0);
    end = (int32_t)min((int64_t)held + max(n, 0), (int64_t)kMostLength);
    return (uint32_t)max(n, 0);
}

// What becomes of an entry.
struct Entry {
    bool there, wanted, takes;
    __device__ __forceinline__ Entry(const TablesArgs &a, uint32_t i, int32_t page, int32_t held, int32_t end)
    {
        const int32_t from = (int32_t)(a.prefix_len + (i << a.page_shift)); // inside the capacity, as the entry is
        there = (uint32_t)page < a.n_pages;
        wanted = from < end;
        if (a.window) wanted = wanted & (((int64_t)from + (1 << a.page_shift) - 1 > (int64_t)held - a.window) | ((uint32_t)from < a.sinks));
        takes = wanted & !there & (from >= held);
    }
};

// A wavefront's entries of run `item`: entry first + 64 k + lane in page[k]; those beyond the row are -2.
__device__ __forceinline__ void load_run(const TablesArgs &a, uint32_t item, uint32_t lane, uint32_t &seq, uint32_t &first, int32_t (&page)[kLoads])
{
    seq = item / a.runs, first = item % a.runs * kRun;
    const int32_t *row = a.pages_in + (uint64_t)seq * a.stride;
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        const uint32_t i = first + 64 * k + lane;
        page[k] = i < a.stride ? row[i] : -2;
    }
}

__device__ __forceinline__ void count_run(const TablesArgs &a, uint32_t item, uint32_t lane)
{
    uint32_t seq, first;
    int32_t page[kLoads], held, end;
    load_run(a, item, lane, seq, first, page);
    tokens_of(a, seq, held, end);
    Moves m = {0, 0};
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        const uint32_t i = first + 64 * k + lane;
        const Entry e(a, min(i, a.stride - 1), page[k], held, end);
        m.taken += (uint32_t)__popcll(__ballot((i < a.stride) & e.takes));
        m.back += (uint32_t)__popcll(__ballot((i < a.stride) & e.there & !e.wanted));
    }
    if (lane == 0) a.ws_moves[item] = m;
}

// Inclusive sums over the threads of a workgroup, and the sum of all; every thread takes part.
template <typename V> __device__ __forceinline__ V workgroup_sums(V v, V &all, V *lds)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const V t = __shfl_up(v, k);
        if (lane >= (uint32_t)k) v += t;
    }
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    V before = 0;
    all = 0;
    for (uint32_t w = 0; w < kScanThreads / 64; w++) {
        const V t = lds[w];
        if (w < wave) before += t;
        all += t;
    }
    __syncthreads();
    return before + v;
}

// Rows of the sequences, and how many moves there are before each run: one workgroup of kScanThreads.
__device__ __forceinline__ void sum_up(const TablesArgs &a, unsigned long long *lds)
{
    unsigned long long rows = 0, all;
    for (uint32_t b = 0; b < a.n_seqs; b += kScanThreads) {
        const uint32_t seq = b + threadIdx.x;
        int32_t held = 0, end = 0;
        const unsigned long long arriving = seq < a.n_seqs ? tokens_of(a, seq, held, end) : 0, upto = rows + workgroup_sums<unsigned long long>(arriving, all, lds);
        if (seq < a.n_seqs) {
            const uint32_t first = (uint32_t)min(upto - arriving, (unsigned long long)a.n_rows), last = (uint32_t)min(upto, (unsigned long long)a.n_rows);
            a.ws_seqs[seq] = Sequence{held, end, first, last - first};
            a.len[seq] = min(end, (int32_t)min((int64_t)held + (last - first), (int64_t)kMostLength));
            a.row_start[seq] = (int32_t)first;
            if (seq == a.n_seqs - 1) a.row_start[a.n_seqs] = (int32_t)last;
        }
        rows += all;
    }
    // both counts in one number: neither reaches 2^31
    unsigned long long moves = 0;
    for (uint32_t b = 0; b < a.n_items; b += kScanThreads) {
        const uint32_t item = b + threadIdx.x;
        unsigned long long v = 0;
        if (item < a.n_items) {
            const Moves m = a.ws_moves[item];
            v = (unsigned long long)m.back << 32 | m.taken;
        }
        const unsigned long long before = moves + workgroup_sums<unsigned long long>(v, all, lds) - v;
        if (item < a.n_items) a.ws_moves[item] = Moves{(uint32_t)before, (uint32_t)(before >> 32)};
        moves += all;
    }
    if (threadIdx.x == 0) {
        const Queue q = {(uint32_t)a.queue_in[0] % a.n_pages, (uint32_t)min((int64_t)max(a.queue_in[1], 0), (int64_t)a.n_pages)};
        *a.ws_queue = q;
        const uint32_t taken = (uint32_t)moves, back = (uint32_t)(moves >> 32), got = min(taken, q.count);
        a.queue[0] = (int32_t)(((uint64_t)q.first + got) % a.n_pages);
        a.queue[1] = (int32_t)min((uint64_t)(q.count - got) + back, (uint64_t)a.n_pages);
        a.queue[2] = (int32_t)(taken - got);
    }
}

// A run's entries as they become, and the places of the rows that lie on them.  lds: address of kRun entries of the wavefront's own.
__device__ __forceinline__ void fill_run(const TablesArgs &a, uint32_t item, uint32_t lane, uint32_t lds)
{
    uint32_t seq, first;
    int32_t page[kLoads];
    load_run(a, item, lane, seq, first, page);
    const Sequence s = a.ws_seqs[seq];
    const Queue q = *a.ws_queue;
    Moves at = a.ws_moves[item];
    const uint64_t below = (1ull << lane) - 1;
    int32_t *row = a.pages + (uint64_t)seq * a.stride;
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        const uint32_t i = first + 64 * k + lane;
        const bool is = i < a.stride;
        const Entry e(a, min(i, a.stride - 1), page[k], s.held, s.end);
        const uint64_t taking = __ballot(is & e.takes), giving = __ballot(is & e.there & !e.wanted);
        const uint32_t rank = at.taken + (uint32_t)__popcll(taking & below), rank_back = at.back + (uint32_t)__popcll(giving & below);
        int32_t p = (e.there & e.wanted) ? page[k] : -1;
        if (is & e.takes & (rank < q.count)) p = a.free[((uint64_t)q.first + rank) % a.n_pages];
        if (is & e.there & !e.wanted) a.free[((uint64_t)q.first + q.count + rank_back) % a.n_pages] = page[k];
        if (is) row[i] = p;
        *(dcdev::lds_u32 *)(uintptr_t)(lds + 4 * (64 * k + lane)) = (uint32_t)p;
        at.taken += (uint32_t)__popcll(taking), at.back += (uint32_t)__popcll(giving);
    }
    __builtin_amdgcn_wave_barrier();
    if (!a.slot && !a.position && !a.seq) return;
    // the sequence's rows from the run's first position on (the first run: from the beginning) to its last (the last run: to the end)
    const int64_t from = first ? (int64_t)a.prefix_len + ((int64_t)first << a.page_shift) : 0;
    const int64_t to = first + kRun < a.stride ? (int64_t)a.prefix_len + ((int64_t)(first + kRun) << a.page_shift) : INT64_MAX;
    const int64_t p_first = max(from, (int64_t)s.held), p_end = min(to, (int64_t)s.held + s.rows);
    for (int64_t pos = p_first + lane; pos < p_end; pos += 64) {
        const uint32_t r = s.first_row + (uint32_t)(pos - s.held), p = (uint32_t)pos;
        const uint32_t place = p < a.prefix_len ? p : p - a.prefix_len, i = place >> a.page_shift;
        int32_t of = -1;
        if (p < a.prefix_len) of = a.prefix_pages[i];
        else if (i < a.stride) of = (int32_t)dcdev::lds_load32(lds + 4 * (i - first));
        const uint32_t in_page = place & ((1u << a.page_shift) - 1u);
        if (a.slot) a.slot[r] = (uint32_t)of < a.n_pages ? ((int64_t)of << a.page_shift) + in_page : -1;
        if (a.position) a.position[r] = (int32_t)min(pos, (int64_t)kMostLength);
        if (a.seq) a.seq[r] = (int32_t)seq;
    }
}

// Rows of no sequence.
__device__ __forceinline__ void fill_rest(const TablesArgs &a, uint32_t thread, uint32_t threads)
{
    const Sequence s = a.ws_seqs[a.n_seqs - 1];
    for (uint64_t r = (uint64_t)s.first_row + s.rows + thread; r < a.n_rows; r += threads) {
        if (a.slot) a.slot[r] = -1;
        if (a.position) a.position[r] = -1;
        if (a.seq) a.seq[r] = -1;
    }
}

__global__ __launch_bounds__(256) void dc_kv_tables_count_kernel(TablesArgs a)
{
    for (uint32_t item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < a.n_items; item += gridDim.x * 4) count_run(a, item, threadIdx.x & 63u);
}

__global__ __launch_bounds__(kScanThreads) void dc_kv_tables_sum_kernel(TablesArgs a)
{
    __shared__ unsigned long long lds[kScanThreads / 64];
    sum_up(a, lds);
}

__global__ __launch_bounds__(256) void dc_kv_tables_fill_kernel(TablesArgs a)
{
    __shared__ int32_t lds[4][kRun];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint32_t item = blockIdx.x * 4 + wave; item < a.n_items; item += gridDim.x * 4) fill_run(a, item, threadIdx.x & 63u, dcdev::lds_address(lds) + wave * (kRun * 4));
    fill_rest(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

__global__ __launch_bounds__(kScanThreads) void dc_kv_tables_kernel(TablesArgs a)
{
    __shared__ int32_t lds[kScanThreads / 64][kRun];
    __shared__ unsigned long long sums[kScanThreads / 64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    for (uint32_t item = wave; item < a.n_items; item += kScanThreads / 64) count_run(a, item, lane);
    __syncthreads();
    sum_up(a, sums);
    __syncthreads();
    for (uint32_t item = wave; item < a.n_items; item += kScanThreads / 64) fill_run(a, item, lane, dcdev::lds_address(lds) + wave * (kRun * 4));
    fill_rest(a, threadIdx.x, kScanThreads);
}

bool requests_ok(const dc_kv_requests *r)
{
    if (!r || r->n_seqs < 1 || r->n_seqs > 65535 || r->n_rows < 1 || r->n_rows >= 1u << 24 || !page_tokens_ok(r->page_tokens) || r->pages_stride < 1 ||
        r->n_pages < 1 || r->n_pages > 0x7FFFFFFFu || (uint64_t)r->n_seqs * r->pages_stride >= 1ull << 31)
        return false;
    if ((r->prefix_len != 0) != (r->prefix_pages_dev != nullptr)) return false;
    if ((uint64_t)r->prefix_len + (uint64_t)r->pages_stride * r->page_tokens > 0x7FFF0000ull) return false;
    const void *needed[] = {r->held_dev, r->new_dev, r->pages_in_dev, r->queue_in_dev, r->free_dev, r->len_dev, r->row_start_dev, r->pages_dev, r->queue_dev};
    for (const void *p : needed)
        if (!p || (uintptr_t)p & 3u) return false;
    return ((uintptr_t)r->prefix_pages_dev & 3u) == 0 && ((uintptr_t)r->position_dev & 3u) == 0 && ((uintptr_t)r->seq_dev & 3u) == 0 &&
           ((uintptr_t)r->slot_dev & 7u) == 0;
}

uint32_t runs_of(const dc_kv_requests *r) { return (r->pages_stride + kRun - 1) / kRun; }
uint64_t workspace_of(const dc_kv_requests *r)
{
    return sizeof(Queue) + sizeof(Sequence) * (uint64_t)r->n_seqs + sizeof(Moves) * (uint64_t)r->n_seqs * runs_of(r);
}

} // namespace

extern "C" int dc_kv_tables_workspace(const dc_kv_requests *requests, uint64_t *workspace_bytes)
{
    if (!workspace_bytes || !requests_ok(requests)) return DC_E_ARG;
    *workspace_bytes = workspace_of(requests);
    return DC_OK;
}

extern "C" int dc_kv_tables(const dc_kv_requests *requests, void *workspace_dev, uint64_t workspace_bytes, void *hip_stream)
{
    if (!requests_ok(requests) || !workspace_dev || !aligned16(workspace_dev)) return DC_E_ARG;
    if (workspace_bytes < workspace_of(requests)) return DC_E_CAP;
    const dc_kv_requests &r = *requests;
    TablesArgs a = {};
    a.held = r.held_dev, a.arriving = r.new_dev, a.pages_in = r.pages_in_dev, a.prefix_pages = r.prefix_pages_dev, a.queue_in = r.queue_in_dev;
    a.free = r.free_dev, a.len = r.len_dev, a.row_start = r.row_start_dev, a.pages = r.pages_dev, a.queue = r.queue_dev;
    a.position = r.position_dev, a.seq = r.seq_dev, a.slot = r.slot_dev;
    a.n_seqs = r.n_seqs, a.n_rows = r.n_rows, a.page_shift = shift_of(r.page_tokens), a.stride = r.pages_stride, a.n_pages = r.n_pages;
    a.prefix_len = r.prefix_len, a.window = r.window, a.sinks = r.sinks, a.runs = runs_of(&r), a.n_items = r.n_seqs * a.runs;
    a.ws_queue = static_cast<Queue *>(workspace_dev);
    a.ws_seqs = reinterpret_cast<Sequence *>(a.ws_queue + 1);
    a.ws_moves = reinterpret_cast<Moves *>(a.ws_seqs + r.n_seqs);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (a.n_items <= kScanThreads / 64) {
        hipLaunchKernelGGL(dc_kv_tables_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
    } else {
        const dim3 grid(std::min<uint32_t>((a.n_items + 3) / 4, 1u << 20));
        hipLaunchKernelGGL(dc_kv_tables_count_kernel, grid, dim3(256), 0, stream, a);
        hipLaunchKernelGGL(dc_kv_tables_sum_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
        hipLaunchKernelGGL(dc_kv_tables_fill_kernel, grid, dim3(256), 0, stream, a);
    }
    return dc_launch_status();
}
