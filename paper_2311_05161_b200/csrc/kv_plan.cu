// A step's plan on the device: from the requests' lengths the page table, row offsets, positions and slots.
//
// Every CTA computes the prefix sums of rows, pages taken and pages given back over the batch (three sums in one scan) into
// its shared memory, so that each can fill its share of the outputs without waiting for another.  The free list is a stack: what
// is given back lies on top of it in the order of sequences and pages, and page number a of those taken is the a-th from the
// top, which every thread finds by itself (on the list, or in the table of the sequence that gives it back).  The lengths and the
// count may be updated in place: a CTA draws a ticket when it has read them, and the one that draws the last writes them.
// A step is taken or refused as a whole, so every CTA looks at all numbers that change hands before it writes: to leave that to the CTA that moves
// a number would mean to wait for one another, or to undo.
//
// Twelve bytes per row and a few per sequence: the time is a launch, the scan's chain of dependent steps, and for many rows
// the search of each row's sequence, which four neighbouring rows share.  Eight requests of a token each 4.1 us; 1500 requests with
// 252 thousand rows, 7900 pages taken and 4000 given back 14.1 us (3.2 MB, 0.5 us of memory; a search and scattered stores for every row took
// 7.5 us more), 4 us of it for the look at the numbers that change hands: 0.5 those from the list, 3.5 those given back, each of which every CTA reads
// from the same lines of L2 behind a search of its sequence (one by one, instead of eight side by side, 8 us).  8000 requests of a token each
// 14.5 us, the scan (45 us where the threads' entries met in one bank).
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kRun = 4;                      // neighbouring rows of a thread
constexpr int kChecked = 8;                  // pages of a thread that are looked at together
constexpr int kAtOnce = 4;                   // sequences of a thread whose lengths are loaded together

struct Sums {
    long long rows, taken, back;
};
__device__ __forceinline__ Sums plus(const Sums &a, const Sums &b) { return {a.rows + b.rows, a.taken + b.taken, a.back + b.back}; }

struct Request {
    int held, kept, add;
    int had, has;                            // pages
    bool good;
    __device__ Sums sums() const { return {good ? add : 0, max(has - had, 0), max(had - has, 0)}; }
};
__device__ __forceinline__ Request load_request(const KvPlanArgs &a, int b)
{
    Request q;
    q.kept = __ldca(a.kv_lens + b);
    q.held = a.held ? __ldca(a.held + b) : q.kept;
    q.add = __ldca(a.add + b);
    return q;
}
__device__ __forceinline__ void count_pages(const KvPlanArgs &a, Request &q)
{
    const long long most = (long long)a.max_pages << a.page_shift;
    q.good = q.kept >= 0 && q.add >= 0 && q.held >= q.kept && q.held <= most && (long long)q.kept + q.add <= most;
    const int round = (1 << a.page_shift) - 1;
    q.had = q.good ? (q.held + round) >> a.page_shift : 0;
    q.has = q.good ? (q.kept + q.add + round) >> a.page_shift : 0;
}

// What the outputs need to know of a sequence.
struct __align__(16) Entry {
    int row, kept, taken, had;               // first row, tokens, first page taken, pages before
};

// The last sequence of lo .. hi whose number is <= x, where numbers ascend and lo's is <= x: the owner of element x.
template <class F>
__device__ __forceinline__ int owner(int lo, int hi, int x, F number)
{
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (number(mid) <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) kv_plan_kernel(const KvPlanArgs a, StatusBlock *sb, int *ticket)
{
    constexpr int WARPS = THREADS / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Sums warp_sums[WARPS];
    __shared__ int last;
    allow_dependents();
    dependent_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = a.batch;
    Entry *entry = reinterpret_cast<Entry *>(smem);                        // [batch]
    int *first_back = reinterpret_cast<int *>(smem + sizeof(Entry) * batch);   // [batch]: first page given back; pages afterwards
    int *pages_left = first_back + batch;
    const int chunk = (batch + THREADS - 1) / THREADS | 1;     // odd: the threads' entries lie in different banks
    const int b0 = min(batch, tid * chunk), b1 = min(batch, b0 + chunk);
    const int count = __ldca(a.free_count);
    Sums mine = {0, 0, 0};
    bool bad = false;
    for (int b = b0; b < b1; b += kAtOnce) {
        Request q[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (b + k < b1) q[k] = load_request(a, b + k);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            if (b + k >= b1) break;
            count_pages(a, q[k]);
            if (!q[k].good) {
                bad = true;
                report_failure(sb, W4A8_ERR_BAD_TABLE, b + k);
            }
            // (sums of this thread's sequences so far; what lies before them is added below)
            entry[b + k] = {(int)mine.rows, q[k].kept, (int)mine.taken, q[k].had};
            first_back[b + k] = (int)mine.back;
            pages_left[b + k] = q[k].has;
            mine = plus(mine, q[k].sums());
        }
    }
    Sums upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums v = {__shfl_up_sync(0xffffffffu, upto.rows, o), __shfl_up_sync(0xffffffffu, upto.taken, o),
                        __shfl_up_sync(0xffffffffu, upto.back, o)};
        if (lane >= o) upto = plus(upto, v);
    }
    if (lane == 31) warp_sums[warp] = upto;
    bad = __syncthreads_or(bad);             // also: this CTA has read the lengths and the count
    int tickets = 0;                         // drawn before this CTA's
    if (tid == 0 && gridDim.x > 1) asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(tickets) : "l"(ticket) : "memory");
    Sums total = {0, 0, 0}, before = {upto.rows - mine.rows, upto.taken - mine.taken, upto.back - mine.back};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        const Sums v = warp_sums[w];
        if (w < warp) before = plus(before, v);
        total = plus(total, v);
    }
    // ---- all or nothing ----
    if (!bad && (total.rows > a.rows || count < 0 || count > a.num_pages || count + total.back > a.num_pages)) {
        bad = true;
        if (tid == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, -1);
    }
    if (!bad && total.taken > count + total.back) {
        bad = true;
        if (tid == 0) report_failure(sb, W4A8_ERR_NO_PAGES, -1);
    }
    for (int b = b0; b < b1; ++b) {
        entry[b].row += (int)before.rows;
        entry[b].taken += (int)before.taken;
        first_back[b] += (int)before.back;
    }
    __syncthreads();
    // page that sequence b gives back as place f
    auto back_page = [&](int b, int f) { return __ldca(a.page_table + (size_t)b * a.max_pages + pages_left[b] + f - first_back[b]); };
    // Every CTA looks at all pages that change hands before it writes anything.  (What it looks at is written by none: table entries in
    // front of `had`, the list below `count`.)
    const int n_popped = bad ? 0 : (int)max(total.taken - total.back, 0ll);      // from the list itself
    if (!bad && (n_popped > 0 || total.back > 0)) {
        int lost = 0;                        // a page number that is none: 1 + its sequence, or -1 (the list)
        int page[kChecked];                  // their loads in flight together
        for (uint32_t k0 = tid; k0 < (uint32_t)n_popped; k0 += kChecked * THREADS) {
#pragma unroll
            for (int k = 0; k < kChecked; ++k) page[k] = k0 + k * THREADS < (uint32_t)n_popped ? __ldca(a.free_pages + count - 1 - (k0 + k * THREADS)) : 0;
#pragma unroll
            for (int k = 0; k < kChecked; ++k)
                if ((unsigned)page[k] >= (unsigned)a.num_pages) lost = -1;
        }
        // A warp takes a part of those given back, its lanes neighbours; they belong to sequences lo .. hi.
        const int all = (int)total.back;
        const long long part = ((all + WARPS - 1) / WARPS + 31) / 32 * 32;
        const int f0 = (int)min((long long)all, warp * part), f1 = (int)min((long long)all, f0 + part);
        if (f0 < f1) {
            const int end = owner(0, batch - 1, lane & 1 ? f1 - 1 : f0, [&](int i) { return first_back[i]; });
            const int lo = __shfl_sync(0xffffffffu, end, 0), hi = __shfl_sync(0xffffffffu, end, 1);
            const int step0 = hi > lo ? 1 << (31 - __clz(hi - lo)) : 0;
            for (int f = f0 + lane; f < f1; f += kChecked * 32) {
                int b[kChecked];
#pragma unroll
                for (int k = 0; k < kChecked; ++k) b[k] = lo;
                for (int step = step0; step > 0; step >>= 1) {             // (side by side)
#pragma unroll
                    for (int k = 0; k < kChecked; ++k)
                        if (b[k] + step <= hi && first_back[b[k] + step] <= f + 32 * k) b[k] += step;
                }
#pragma unroll
                for (int k = 0; k < kChecked; ++k) page[k] = f + 32 * k < f1 ? back_page(b[k], f + 32 * k) : 0;
#pragma unroll
                for (int k = 0; k < kChecked; ++k)
                    if ((unsigned)page[k] >= (unsigned)a.num_pages) lost = b[k] + 1;
            }
        }
        if (lost) report_failure(sb, W4A8_ERR_BAD_TABLE, lost > 0 ? lost - 1 : -2);
        bad = __syncthreads_or(lost);
    }
    const int n_rows = bad ? 0 : (int)total.rows, n_taken = bad ? 0 : (int)total.taken, n_back = bad ? 0 : (int)total.back;
    const int top = count + n_back;          // of the stack with what is given back
    if (blockIdx.x == 0) {
        for (int b = tid; b < batch; b += THREADS) a.cu_rows[b] = bad ? 0 : entry[b].row;
        if (tid == 0) a.cu_rows[batch] = n_rows;
    }
    // page of place f among those given back, and of place k from the top of the stack
    auto given_back = [&](int f) { return back_page(owner(0, batch - 1, f, [&](int i) { return first_back[i]; }), f); };
    auto taken = [&](int k) {
        const int v = top - 1 - k;
        return v < count ? __ldca(a.free_pages + v) : given_back(v - count);
    };
    const int thread = blockIdx.x * THREADS + tid, threads = gridDim.x * THREADS;
    // (pages from the last thread on, rows from the first)
    for (int k = threads - 1 - thread; k < n_taken; k += threads) {
        const int b = owner(0, batch - 1, k, [&](int i) { return entry[i].taken; });
        a.page_table[(size_t)b * a.max_pages + entry[b].had + k - entry[b].taken] = taken(k);
    }
    for (int f = threads - 1 - thread; f < n_back - n_taken; f += threads) a.free_pages[count + f] = given_back(f);
    for (int r0 = thread * kRun; r0 < a.rows && (a.positions || a.slots); r0 += threads * kRun) {
        int pos[kRun];
        long long slot[kRun];
        int b = r0 < n_rows ? owner(0, batch - 1, r0, [&](int i) { return entry[i].row; }) : batch;
        int at = -1, page = 0;               // the page looked up last
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            pos[k] = 0;
            slot[k] = -1;
            if (r0 + k >= n_rows) continue;
            while (b + 1 < batch && entry[b + 1].row <= r0 + k) {
                ++b;
                at = -1;
            }
            const Entry e = entry[b];
            pos[k] = e.kept + r0 + k - e.row;
            const int i = pos[k] >> a.page_shift;
            if (i != at) {
                at = i;
                page = i < e.had ? __ldca(a.page_table + (size_t)b * a.max_pages + i) : taken(e.taken + i - e.had);
                if ((unsigned)page >= (unsigned)a.num_pages) report_failure(sb, W4A8_ERR_BAD_TABLE, b);      // the table lost it
            }
            if ((unsigned)page < (unsigned)a.num_pages) slot[k] = ((long long)page << a.page_shift) + (pos[k] & ((1 << a.page_shift) - 1));
        }
        if (r0 + kRun <= a.rows && a.wide_stores) {
            if (a.positions) *reinterpret_cast<int4 *>(a.positions + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            if (a.slots) {
                longlong2 *to = reinterpret_cast<longlong2 *>(a.slots + r0);
                to[0] = make_longlong2(slot[0], slot[1]);
                to[1] = make_longlong2(slot[2], slot[3]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                if (r0 + k >= a.rows) break;
                if (a.positions) a.positions[r0 + k] = pos[k];
                if (a.slots) a.slots[r0 + k] = slot[k];
            }
        }
    }
    // ---- lengths and count, by the CTA with the last ticket ----
    if (tid == 0) last = tickets == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    for (int b = tid; b < batch; b += THREADS) {
        const Request q = load_request(a, b);
        a.kv_lens_out[b] = bad ? q.held : q.kept + q.add;
    }
    if (tid == 0) {
        *a.free_count_out = top - n_taken;
        *ticket = 0;                         // ready for the next call
    }
}

template <int THREADS>
cudaError_t launch(const KvPlanArgs &a, StatusBlock *sb, int *ticket, cudaStream_t st)
{
    const int smem = (int)(sizeof(Entry) + 2 * sizeof(int)) * a.batch;
    static std::atomic<int> raised[kMaxDevices];
    const cudaError_t e = raise_smem_limit(kv_plan_kernel<THREADS>, smem, raised);
    if (e != cudaSuccess) return e;
    // a thread for every run of rows, and for every page that so many rows of so many sequences may need
    const long long threads = (a.rows + kRun - 1) / kRun + (a.rows >> a.page_shift) + (a.batch > THREADS ? a.batch : 0);
    const long long ctas = (threads + THREADS - 1) / THREADS, sms = device_sms();
    return launch_overlapped(kv_plan_kernel<THREADS>, dim3((unsigned)(ctas < sms ? ctas : sms)), dim3(THREADS), smem, st, a, sb, ticket);
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanArgs &args, StatusBlock *sb, int *ticket, cudaStream_t st)
{
    KvPlanArgs a = args;
    a.wide_stores = reinterpret_cast<uintptr_t>(a.positions) % 16 == 0 && reinterpret_cast<uintptr_t>(a.slots) % 16 == 0;
    // a decode step fits one small CTA, whose barriers and sums are short
    return a.batch <= 128 && a.rows <= 128 * kRun ? launch<128>(a, sb, ticket, st) : launch<512>(a, sb, ticket, st);
}

}  // namespace w4a8
