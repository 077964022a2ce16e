// A step's tables from the tokens that sequences hold and get: lengths, first rows, pages taken and given back, and each row's place.
//
// Pages are taken and given back in the order of sequences and entries, so an entry's place in the queue is the number of entries before it that
// take (give back) a page: counts, their prefix sums, and the entries once more.  A wavefront works on a run of neighbouring entries of one
// sequence; few runs are one workgroup's (one sequence of 64 entries 4.3 us), more take a launch for the counts and one for the results (256 sequences of
// 512 entries 8.4 us, 1024 of 1024 with 215616 rows 12.1 us), and from 16384 runs on one for the sums between them.  Latency bounds all of it: launches, and
// in each a few loads that wait for one another; what the largest of those reads and writes would take 1.8 us.
#include "dc_device.h"
#include "dc_pages.h"

#include <algorithm>

using namespace dcpages;

namespace {

constexpr uint32_t kLoads = 4, kRun = 64 * kLoads; // entries of a run
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
// Entries of a run that take a page, and that give one back; or of all runs before it.
struct Moves {
    uint32_t taken, back;
};

// Of 4 neighbouring runs: their moves, and the rows of the sequences that end among them (2^25 for all that are more).
struct Group {
    uint32_t taken, back, rows, unused;
};
constexpr uint32_t kManyRows = 1u << 25; // more than row arrays can have; sums of a few of them stay inside 32 bits

struct TablesArgs {
    const int32_t *held, *arriving, *pages_in, *prefix_pages, *queue_in;
    int32_t *free, *len, *row_start, *pages, *queue, *position, *seq;
    int64_t *slot;
    Queue *ws_queue;
    Sequence *ws_seqs;
    struct Group *ws_groups;
    Moves *ws_moves;
    uint32_t n_seqs, n_rows, page_shift, stride, n_pages, prefix_len, window, sinks;
    uint32_t runs, n_items; // runs of a sequence, of all
};

// Tokens that a sequence holds, and with all the new ones.
__device__ __forceinline__ uint32_t arriving_at(const TablesArgs &a, uint32_t seq) { return (uint32_t)max(a.arriving[seq], 0); }
__device__ __forceinline__ void tokens_of(const TablesArgs &a, uint32_t seq, int32_t &held, int32_t &end)
{
    const int32_t n = a.arriving[seq], h = a.held[seq];
    held = n < 0 ? 0 : max(h, 0);
    end = (int32_t)min((int64_t)held + max(n, 0), (int64_t)kMostLength);
}
__device__ __forceinline__ Queue queue_of(const TablesArgs &a)
{
    return Queue{(uint32_t)a.queue_in[0] % a.n_pages, (uint32_t)min((int64_t)max(a.queue_in[1], 0), (int64_t)a.n_pages)};
}

// What becomes of an entry.
struct Entry {
    bool there, wanted, takes, goes;
    __device__ __forceinline__ Entry(const TablesArgs &a, uint32_t i, int32_t page, int32_t held, int32_t end)
    {
        const bool is = i < a.stride;
        const int32_t from = (int32_t)(a.prefix_len + (i << a.page_shift)); // inside the capacity, as the entry is
        there = is & ((uint32_t)page < a.n_pages);
        wanted = from < end;
        if (a.window) wanted = wanted & (((int64_t)from + (1 << a.page_shift) - 1 > (int64_t)held - a.window) | ((uint32_t)from < a.sinks));
        takes = is & wanted & !there & (from >= held);
        goes = there & !wanted;
    }
};

// A wavefront's entries of run `item`: entry first + 64 k + lane in page[k].
__device__ __forceinline__ void load_run(const TablesArgs &a, uint32_t item, uint32_t lane, uint32_t &seq, uint32_t &first, int32_t (&page)[kLoads])
{
    seq = item / a.runs, first = item % a.runs * kRun;
    const int32_t *row = a.pages_in + (uint64_t)seq * a.stride;
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        const uint32_t i = first + 64 * k + lane;
        page[k] = -1;
        if (i < a.stride) page[k] = row[i];
    }
}

__device__ __forceinline__ Moves moves_of(const TablesArgs &a, uint32_t first, uint32_t lane, const int32_t (&page)[kLoads], int32_t held, int32_t end)
{
    Moves m = {0, 0};
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        if (first + 64 * k >= a.stride) break;
        const Entry e(a, first + 64 * k + lane, page[k], held, end);
        m.taken += (uint32_t)__popcll(__ballot(e.takes));
        m.back += (uint32_t)__popcll(__ballot(e.goes));
    }
    return m;
}

// Inclusive sums over the threads of a workgroup, and the sum of all; every thread takes part.
template <uint32_t WAVES, typename V> __device__ __forceinline__ V workgroup_sums(V v, V &all, V *lds)
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
#pragma unroll
    for (uint32_t w = 0; w < WAVES; w++) {
        const V t = lds[w];
        if (w < wave) before += t;
        all += t;
    }
    __syncthreads();
    return before + v;
}
typedef unsigned long long u64;
// Both counts of moves in one number: neither reaches 2^31.
__device__ __forceinline__ u64 packed(Moves m) { return (u64)m.back << 32 | m.taken; }
__device__ __forceinline__ Moves unpacked(u64 v) { return Moves{(uint32_t)v, (uint32_t)(v >> 32)}; }

// A sequence's rows, of which `before` are those of the sequences before it; and its results.
__device__ __forceinline__ Sequence sequence_from(const TablesArgs &a, uint32_t seq, int32_t held, int32_t end, u64 before, uint32_t arriving)
{
    const uint32_t first = (uint32_t)min(before, (u64)a.n_rows), last = (uint32_t)min(before + arriving, (u64)a.n_rows);
    return Sequence{held, end, first, last - first};
}
__device__ __forceinline__ void store_sequence(const TablesArgs &a, uint32_t seq, const Sequence &s)
{
    a.len[seq] = min(s.end, (int32_t)min((int64_t)s.held + s.rows, (int64_t)kMostLength));
    a.row_start[seq] = (int32_t)s.first_row;
    if (seq == a.n_seqs - 1) a.row_start[a.n_seqs] = (int32_t)(s.first_row + s.rows);
}
__device__ __forceinline__ void store_queue(const TablesArgs &a, const Queue &q, Moves m)
{
    const uint32_t got = min(m.taken, q.count);
    a.queue[0] = (int32_t)(((u64)q.first + got) % a.n_pages);
    a.queue[1] = (int32_t)min((u64)(q.count - got) + m.back, (u64)a.n_pages);
    a.queue[2] = (int32_t)(m.taken - got);
}

// Rows of a sequence that lie on a run's entries: positions begin .. end - 1, whose rows are less + position.
struct RunRows {
    uint32_t seq, first, begin, end, less;
};

// A run's entries as they become.  at: moves of the runs before.
__device__ __forceinline__ void entries_of(const TablesArgs &a, uint32_t first, uint32_t lane, const int32_t (&page)[kLoads], int32_t held, int32_t end_token, const Queue &q,
                                           Moves at, int32_t (&becomes)[kLoads])
{
    const uint64_t below = (1ull << lane) - 1;
    // places in the ring: sums of two numbers up to n_pages stay inside 32 bits
    auto in_ring = [&](uint32_t x) { return x >= a.n_pages ? x - a.n_pages : x; };
    const uint32_t end = in_ring(q.first + q.count);
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        becomes[k] = -1;
        if (first + 64 * k >= a.stride) break;
        const Entry e(a, first + 64 * k + lane, page[k], held, end_token);
        const uint64_t taking = __ballot(e.takes), giving = __ballot(e.goes);
        const uint32_t rank = at.taken + (uint32_t)__popcll(taking & below), rank_back = at.back + (uint32_t)__popcll(giving & below);
        if (e.there & e.wanted) becomes[k] = page[k];
        if (e.takes & (rank < q.count)) becomes[k] = a.free[in_ring(q.first + rank)];
        if (e.goes & (rank_back < a.n_pages)) a.free[in_ring(end + rank_back)] = page[k];
        at.taken += (uint32_t)__popcll(taking), at.back += (uint32_t)__popcll(giving);
    }
}
// Stores them, also to the kRun entries of the run in the LDS, at address lds; and which rows lie on them.
__device__ __forceinline__ void store_run(const TablesArgs &a, uint32_t seq, uint32_t first, uint32_t lane, const int32_t (&becomes)[kLoads], const Sequence &s, uint32_t lds, RunRows &rows)
{
    int32_t *row = a.pages + (uint64_t)seq * a.stride;
#pragma unroll
    for (uint32_t k = 0; k < kLoads; k++) {
        if (first + 64 * k >= a.stride) break;
        if (first + 64 * k + lane < a.stride) row[first + 64 * k + lane] = becomes[k];
        *(dcdev::lds_u32 *)(uintptr_t)(lds + 4 * (64 * k + lane)) = (uint32_t)becomes[k];
    }
    if (lane == 0) {
        // the sequence's rows from the run's first position on (the first run: from the beginning) to its last (the last run: to the end)
        const uint32_t from = first ? a.prefix_len + (first << a.page_shift) : 0;
        const uint32_t to = first + kRun < a.stride ? a.prefix_len + ((first + kRun) << a.page_shift) : 0xFFFFFFFFu;
        const uint32_t begin = max(from, (uint32_t)s.held), end = min(to, (uint32_t)s.held + s.rows);
        rows = RunRows{seq, first, begin, begin < end ? end : begin, s.first_row - (uint32_t)s.held};
    }
}
__device__ __forceinline__ void fill_run(const TablesArgs &a, uint32_t seq, uint32_t first, uint32_t lane, const int32_t (&page)[kLoads], const Sequence &s, const Queue &q,
                                         Moves at, uint32_t lds, RunRows &rows)
{
    int32_t becomes[kLoads];
    entries_of(a, first, lane, page, s.held, s.end, q, at, becomes);
    store_run(a, seq, first, lane, becomes, s, lds, rows);
}

// The places of the rows that lie on a run's entries: those of number `from`, `from` + STEP ..
template <uint32_t STEP> __device__ __forceinline__ void fill_rows(const TablesArgs &a, const RunRows &rows, uint32_t lds, uint32_t from, uint32_t most = 0xFFFFFFFFu)
{
    const RunRows n = rows;
    for (uint32_t i = from; i < min(n.end - n.begin, most); i += STEP) {
        const uint32_t p = n.begin + i, r = n.less + p, place = p < a.prefix_len ? p : p - a.prefix_len, e = place >> a.page_shift;
        int32_t of = -1;
        if (p < a.prefix_len) of = a.prefix_pages[e];
        else if (e < a.stride) of = (int32_t)dcdev::lds_load32(lds + 4 * (e - n.first));
        if (a.slot) a.slot[r] = (uint32_t)of < a.n_pages ? (int64_t)((uint64_t)(uint32_t)of << a.page_shift | (place & ((1u << a.page_shift) - 1u))) : -1;
        if (a.position) a.position[r] = (int32_t)min(p, (uint32_t)kMostLength);
        if (a.seq) a.seq[r] = (int32_t)n.seq;
    }
}

// Rows of no sequence, from row `from` on.
__device__ __forceinline__ void fill_rest(const TablesArgs &a, uint32_t from, uint32_t thread, uint32_t threads)
{
    for (u64 r = (u64)from + thread; r < a.n_rows; r += threads) {
        if (a.slot) a.slot[r] = -1;
        if (a.position) a.position[r] = -1;
        if (a.seq) a.seq[r] = -1;
    }
}

// Up to 32 runs: one workgroup with RUNS of them to a wavefront, number wave + 16 k; what one part finds stays in registers and in the LDS.
// (32 sequences of 64 entries 6.2 us, of 256 9.0; in two launches 8.3 and 9.1.  64 runs of 128 entries are 11.5 in one workgroup, whose operations bound it then, and 8.6.)
constexpr uint32_t kWaves = kScanThreads / 64, kFewItems = 32;
template <uint32_t RUNS> __global__ __launch_bounds__(kScanThreads) void dc_kv_tables_kernel(TablesArgs a)
{
    constexpr uint32_t kItems = RUNS * kWaves;
    __shared__ int32_t entries[kItems][kRun];
    __shared__ Moves moves[kItems];
    __shared__ RunRows run_rows[kItems];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    // every wavefront knows all sequences (at most 32): a lane to a sequence
    const uint32_t arriving = lane < a.n_seqs ? arriving_at(a, lane) : 0;
    const Queue q = queue_of(a);
    uint32_t seq[RUNS], first[RUNS];
    int32_t page[RUNS][kLoads], held[RUNS], end[RUNS];
    int32_t lane_held = 0, lane_end = 0;
    if (lane < a.n_seqs) tokens_of(a, lane, lane_held, lane_end);
    // (loads without branches between them: all are under way at once; where there is no such run, the last one's)
#pragma unroll
    for (uint32_t k = 0; k < RUNS; k++) load_run(a, min(wave + kWaves * k, a.n_items - 1), lane, seq[k], first[k], page[k]);
#pragma unroll
    for (uint32_t k = 0; k < RUNS; k++) {
        held[k] = __builtin_amdgcn_readlane(lane_held, (int)seq[k]), end[k] = __builtin_amdgcn_readlane(lane_end, (int)seq[k]);
        Moves mine = {0, 0};
        if (wave + kWaves * k < a.n_items) mine = moves_of(a, first[k], lane, page[k], held[k], end[k]);
        if (lane == 0) moves[wave + kWaves * k] = mine;
    }
    u64 rows_upto = arriving;
#pragma unroll
    for (int k = 1; k < (int)kItems; k <<= 1) {
        const u64 t = __shfl_up(rows_upto, k);
        if (lane >= (uint32_t)k) rows_upto += t;
    }
    const u64 rows = __shfl(rows_upto, kItems - 1);
    __syncthreads(); // (behind it nobody reads what the results may lie on: lengths, queue, entries)
    // moves of the runs before the lane's, and of all
    Moves mine = {0, 0};
    if (lane < kItems) mine = moves[lane];
    const uint32_t taken = dcdev::lanes_prefix_sum<false>(mine.taken), back = dcdev::lanes_prefix_sum<false>(mine.back);
    if (threadIdx.x == 63) store_queue(a, q, Moves{taken, back});
    const uint32_t lds = dcdev::lds_address(entries);
    int32_t becomes[RUNS][kLoads];
#pragma unroll
    for (uint32_t k = 0; k < RUNS; k++) {
        const uint32_t item = wave + kWaves * k;
        if (item >= a.n_items) break;
        const Moves at = {(uint32_t)__builtin_amdgcn_readlane((int)(taken - mine.taken), (int)item), (uint32_t)__builtin_amdgcn_readlane((int)(back - mine.back), (int)item)};
        entries_of(a, first[k], lane, page[k], held[k], end[k], q, at, becomes[k]);
    }
#pragma unroll
    for (uint32_t k = 0; k < RUNS; k++) {
        const uint32_t item = wave + kWaves * k;
        if (item >= a.n_items) break;
        const Sequence s = sequence_from(a, seq[k], held[k], end[k], __shfl(rows_upto - arriving, (int)seq[k]), (uint32_t)__shfl((int)arriving, (int)seq[k]));
        if (lane == 0 && first[k] == 0) store_sequence(a, seq[k], s);
        store_run(a, seq[k], first[k], lane, becomes[k], s, lds + item * (kRun * 4), run_rows[item]);
    }
    fill_rest(a, (uint32_t)min(rows, (u64)a.n_rows), threadIdx.x, kScanThreads);
    __syncthreads();
    // a run's rows: the first ones by its wavefront, further ones by all
#pragma unroll
    for (uint32_t k = 0; k < RUNS; k++) {
        const uint32_t item = wave + kWaves * k;
        if (item < a.n_items) fill_rows<64>(a, run_rows[item], lds + item * (kRun * 4), lane, 64);
    }
    bool more = false;
    if (lane < a.n_items) more = run_rows[lane].end - run_rows[lane].begin > 64;
    uint64_t longer = __ballot(more);
    while (longer) {
        const uint32_t i = (uint32_t)__builtin_ctzll(longer);
        longer &= longer - 1;
        fill_rows<kScanThreads>(a, run_rows[i], lds + i * (kRun * 4), 64 + threadIdx.x);
    }
}

// More: counts of all runs and what the results may lie on, ..
__global__ __launch_bounds__(256) void dc_kv_tables_count_kernel(TablesArgs a)
{
    __shared__ Group runs[4];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ws_queue = queue_of(a);
    for (uint32_t item0 = blockIdx.x * 4; item0 < a.n_items; item0 += gridDim.x * 4) {
        const uint32_t item = item0 + wave;
        Group mine = {};
        if (item < a.n_items) {
            uint32_t seq, first;
            int32_t page[kLoads], held, end;
            load_run(a, item, lane, seq, first, page);
            tokens_of(a, seq, held, end);
            const Moves m = moves_of(a, first, lane, page, held, end);
            const uint32_t rows = arriving_at(a, seq);
            if (lane == 0) a.ws_moves[item] = m;
            if (lane == 0 && first == 0) a.ws_seqs[seq] = Sequence{held, end, 0, rows};
            mine = Group{m.taken, m.back, item % a.runs == a.runs - 1 ? min(rows, kManyRows) : 0u, 0};
        }
        if (lane == 0) runs[wave] = mine;
        __syncthreads();
        if (threadIdx.x == 0) {
            Group g = {};
#pragma unroll
            for (int w = 0; w < 4; w++) g.taken += runs[w].taken, g.back += runs[w].back, g.rows += runs[w].rows;
            g.rows = min(g.rows, kManyRows);
            a.ws_groups[item0 / 4] = g;
        }
        __syncthreads();
    }
}

// .. their sums, if their groups are too many for everyone to add up those before its own ..
constexpr uint32_t kManyItems = 16384;
__global__ __launch_bounds__(kScanThreads) void dc_kv_tables_sum_kernel(TablesArgs a)
{
    __shared__ u64 lds[kScanThreads / 64];
    u64 rows = 0, all;
    for (uint32_t b = 0; b < a.n_seqs; b += kScanThreads) {
        const uint32_t seq = b + threadIdx.x;
        Sequence s = {};
        if (seq < a.n_seqs) s = a.ws_seqs[seq];
        const u64 upto = rows + workgroup_sums<kScanThreads / 64, u64>(s.rows, all, lds);
        if (seq < a.n_seqs) a.ws_seqs[seq] = sequence_from(a, seq, s.held, s.end, upto - s.rows, s.rows);
        rows += all;
    }
    u64 moves = 0;
    for (uint32_t b = 0; b < a.n_items; b += kScanThreads) {
        const uint32_t item = b + threadIdx.x;
        const u64 v = item < a.n_items ? packed(a.ws_moves[item]) : 0;
        const u64 before = moves + workgroup_sums<kScanThreads / 64, u64>(v, all, lds) - v;
        if (item < a.n_items) a.ws_moves[item] = unpacked(before);
        moves += all;
    }
    if (threadIdx.x == 0) store_queue(a, *a.ws_queue, unpacked(moves));
}

// .. and the results.  SUMMED: the sums are there; else a workgroup adds up what its own group has before it.
template <bool SUMMED> __global__ __launch_bounds__(256) void dc_kv_tables_fill_kernel(TablesArgs a)
{
    __shared__ int32_t lds[4][kRun];
    __shared__ uint32_t sums[4][6];
    __shared__ RunRows run_rows[4];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u, address = dcdev::lds_address(lds) + wave * (kRun * 4);
    const Queue q = *a.ws_queue;
    if (SUMMED) {
        for (uint32_t item0 = blockIdx.x * 4; item0 < a.n_items; item0 += gridDim.x * 4) {
            const uint32_t item = item0 + wave;
            if (item < a.n_items) {
                uint32_t seq, first;
                int32_t page[kLoads];
                load_run(a, item, lane, seq, first, page);
                const Sequence s = a.ws_seqs[seq];
                if (lane == 0 && first == 0) store_sequence(a, seq, s);
                fill_run(a, seq, first, lane, page, s, q, a.ws_moves[item], address, run_rows[wave]);
            }
            __syncthreads();
            for (uint32_t i = 0; i < min(4u, a.n_items - item0); i++) fill_rows<256>(a, run_rows[i], dcdev::lds_address(lds) + i * (kRun * 4), threadIdx.x);
            __syncthreads();
        }
        const Sequence s = a.ws_seqs[a.n_seqs - 1];
        fill_rest(a, s.first_row + s.rows, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
        return;
    }
    const uint32_t item = blockIdx.x * 4 + wave; // the grid has a wavefront for each
    uint32_t seq = 0, first = 0;
    int32_t page[kLoads];
    Sequence s = {};
    if (item < a.n_items) {
        load_run(a, item, lane, seq, first, page);
        s = a.ws_seqs[seq];
    }
    // the runs of the workgroup's own group: each in the lanes with its number modulo 4
    const uint32_t item0 = blockIdx.x * 4, groups = (a.n_items + 3) / 4, near = item0 + (lane & 3u);
    Moves near_moves = {0, 0};
    uint32_t near_rows = 0;
    if (near < a.n_items) {
        near_moves = a.ws_moves[near];
        if (near % a.runs == a.runs - 1) near_rows = a.ws_seqs[near / a.runs].rows;
    }
    // moves and rows of all groups of runs, and of those before the workgroup's
    uint32_t mine[6] = {};
    for (uint32_t i = threadIdx.x; i < groups; i += 256) {
        const Group g = a.ws_groups[i];
        mine[3] += g.taken, mine[4] += g.back, mine[5] = min(mine[5] + g.rows, kManyRows);
        if (i < blockIdx.x) mine[0] += g.taken, mine[1] += g.back, mine[2] = min(mine[2] + g.rows, kManyRows);
    }
#pragma unroll
    for (int i = 0; i < 6; i++) {
        const uint32_t v = dcdev::lanes_prefix_sum<false>(mine[i]);
        if (lane == 63) sums[wave][i] = i % 3 == 2 ? min(v, kManyRows) : v;
    }
    __syncthreads();
    uint32_t total[6] = {};
#pragma unroll
    for (int w = 0; w < 4; w++)
#pragma unroll
        for (int i = 0; i < 6; i++) total[i] += sums[w][i];
    if (item == 0 && lane == 0) store_queue(a, q, Moves{total[3], total[4]});
    if (item < a.n_items) {
        Moves at = {total[0], total[1]};
        u64 rows = total[2];
#pragma unroll
        for (uint32_t w = 0; w < 3; w++) { // its own group's runs before it
            if (w >= wave) break;
            at.taken += (uint32_t)__builtin_amdgcn_readlane((int)near_moves.taken, (int)w), at.back += (uint32_t)__builtin_amdgcn_readlane((int)near_moves.back, (int)w);
            rows += (uint32_t)__builtin_amdgcn_readlane((int)near_rows, (int)w);
        }
        s = sequence_from(a, seq, s.held, s.end, rows, s.rows);
        if (lane == 0 && first == 0) store_sequence(a, seq, s);
        fill_run(a, seq, first, lane, page, s, q, at, address, run_rows[wave]);
    }
    fill_rest(a, min(total[5], a.n_rows), blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
    __syncthreads();
    for (uint32_t i = 0; i < min(4u, a.n_items - item0); i++) fill_rows<256>(a, run_rows[i], dcdev::lds_address(lds) + i * (kRun * 4), threadIdx.x);
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
    const uint64_t items = (uint64_t)r->n_seqs * runs_of(r);
    return 16 + sizeof(Sequence) * (uint64_t)r->n_seqs + sizeof(Group) * ((items + 3) / 4) + sizeof(Moves) * items;
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
    a.ws_seqs = reinterpret_cast<Sequence *>(a.ws_queue + 2); // at 16 bytes
    a.ws_groups = reinterpret_cast<Group *>(a.ws_seqs + r.n_seqs);
    a.ws_moves = reinterpret_cast<Moves *>(a.ws_groups + (a.n_items + 3) / 4);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (a.n_items <= kWaves) {
        hipLaunchKernelGGL(dc_kv_tables_kernel<1>, dim3(1), dim3(kScanThreads), 0, stream, a);
    } else if (a.n_items <= kFewItems) {
        hipLaunchKernelGGL(dc_kv_tables_kernel<kFewItems / kWaves>, dim3(1), dim3(kScanThreads), 0, stream, a);
    } else {
        const dim3 grid(std::min<uint32_t>((a.n_items + 3) / 4, 1u << 20));
        hipLaunchKernelGGL(dc_kv_tables_count_kernel, grid, dim3(256), 0, stream, a);
        if (a.n_items <= kManyItems) {
            hipLaunchKernelGGL(dc_kv_tables_fill_kernel<false>, grid, dim3(256), 0, stream, a);
        } else {
            hipLaunchKernelGGL(dc_kv_tables_sum_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
            hipLaunchKernelGGL(dc_kv_tables_fill_kernel<true>, grid, dim3(256), 0, stream, a);
        }
    }
    return dc_launch_status();
}
