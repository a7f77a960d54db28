// A step's plan on the device: from the requests' lengths the page table, row offsets, positions and slots.
//
// Every CTA computes the prefix sums of rows, pages taken and pages given back over the batch (three sums in one scan), so that each
// can fill its share of the outputs by binary search without waiting for another.  The free list is a stack: what is given back
// lies on top of it in the order of sequences and pages, and page number a of those taken is the a-th from the top, which
// every thread finds by itself (on the list, or in the table of the sequence that gives it back).  The lengths and the
// count may be updated in place, so they are written by the CTA that finishes last, when all others have read them.
//
// Twelve bytes per row and a few per sequence: the time is a launch, the scan's chain of dependent steps, and for many rows
// their stores.
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

struct Sums {
    long long rows, taken, back;
};
__device__ __forceinline__ Sums plus(const Sums &a, const Sums &b) { return {a.rows + b.rows, a.taken + b.taken, a.back + b.back}; }

struct Request {
    int held, kept, add;
    int had, has;                            // pages
    bool good;
};
__device__ __forceinline__ Request load_request(const KvPlanArgs &a, int b)
{
    Request q;
    q.kept = __ldca(a.kv_lens + b);
    q.held = a.held ? __ldca(a.held + b) : q.kept;
    q.add = __ldca(a.add + b);
    const long long most = (long long)a.max_pages << a.page_shift;
    q.good = q.kept >= 0 && q.add >= 0 && q.held >= q.kept && q.held <= most && (long long)q.kept + q.add <= most;
    const int round = (1 << a.page_shift) - 1;
    q.had = q.good ? (q.held + round) >> a.page_shift : 0;
    q.has = q.good ? (q.kept + q.add + round) >> a.page_shift : 0;
    return q;
}

// The last of ends[0 .. n] (ascending from 0) that is <= x: the sequence with element x.
__device__ __forceinline__ int owner(const int *ends, int n, int x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (ends[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kThreads) kv_plan_kernel(const KvPlanArgs a, StatusBlock *sb, int *ticket)
{
    extern __shared__ int first[];           // [3][batch]: first row, first page taken, first page given back
    __shared__ Sums warp_sums[kWarps];
    __shared__ int last;
    allow_dependents();
    dependent_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = a.batch;
    int *first_row = first, *first_taken = first + batch, *first_back = first + 2 * batch;
    const int chunk = (batch + kThreads - 1) / kThreads;
    const int b0 = min(batch, tid * chunk), b1 = min(batch, b0 + chunk);
    Sums mine = {0, 0, 0};
    bool bad = false;
    for (int b = b0; b < b1; ++b) {
        const Request q = load_request(a, b);
        bad |= !q.good;
        if (!q.good) report_failure(sb, W4A8_ERR_BAD_TABLE, b);
        mine = plus(mine, {q.good ? q.add : 0, max(q.has - q.had, 0), max(q.had - q.has, 0)});
    }
    Sums upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums v = {__shfl_up_sync(0xffffffffu, upto.rows, o), __shfl_up_sync(0xffffffffu, upto.taken, o),
                        __shfl_up_sync(0xffffffffu, upto.back, o)};
        if (lane >= o) upto = plus(upto, v);
    }
    if (lane == 31) warp_sums[warp] = upto;
    const int count = __ldca(a.free_count);
    bad = __syncthreads_or(bad);
    Sums total = {0, 0, 0};
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto = plus(upto, warp_sums[w]);
        total = plus(total, warp_sums[w]);
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
    const int n_rows = bad ? 0 : (int)total.rows, n_taken = bad ? 0 : (int)total.taken, n_back = bad ? 0 : (int)total.back;
    const int top = count + n_back;          // of the stack with what is given back
    Sums at = {upto.rows - mine.rows, upto.taken - mine.taken, upto.back - mine.back};
    for (int b = b0; b < b1; ++b) {
        first_row[b] = bad ? 0 : (int)at.rows;
        first_taken[b] = bad ? 0 : (int)at.taken;
        first_back[b] = bad ? 0 : (int)at.back;
        if (blockIdx.x == 0) a.cu_rows[b] = first_row[b];
        const Request q = load_request(a, b);
        at = plus(at, {q.add, max(q.has - q.had, 0), max(q.had - q.has, 0)});
    }
    if (blockIdx.x == 0 && tid == 0) a.cu_rows[batch] = n_rows;
    __syncthreads();
    // page of place f among those given back, and of place k from the top of the stack
    auto given_back = [&](int f) {
        const int b = owner(first_back, batch, f);
        return __ldca(a.page_table + (size_t)b * a.max_pages + load_request(a, b).has + f - first_back[b]);
    };
    auto taken = [&](int k) {
        const int v = top - 1 - k;
        const int page = v < count ? __ldca(a.free_pages + v) : given_back(v - count);
        if ((unsigned)page >= (unsigned)a.num_pages) report_failure(sb, W4A8_ERR_BAD_TABLE, -2);
        return page;
    };
    const int thread = blockIdx.x * kThreads + tid, threads = gridDim.x * kThreads;
    for (int k = thread; k < n_taken; k += threads) {
        const int b = owner(first_taken, batch, k);
        a.page_table[(size_t)b * a.max_pages + load_request(a, b).had + k - first_taken[b]] = taken(k);
    }
    for (int f = thread; f < n_back - n_taken; f += threads) a.free_pages[count + f] = given_back(f);
    if (a.positions || a.slots) {
        for (int r = thread; r < a.rows; r += threads) {
            int pos = 0;
            long long slot = -1;
            if (r < n_rows) {
                const int b = owner(first_row, batch, r);
                const Request q = load_request(a, b);
                pos = q.kept + r - first_row[b];
                const int i = pos >> a.page_shift;
                const int page = i < q.had ? __ldca(a.page_table + (size_t)b * a.max_pages + i) : taken(first_taken[b] + i - q.had);
                if ((unsigned)page < (unsigned)a.num_pages) slot = ((long long)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
                else report_failure(sb, W4A8_ERR_BAD_TABLE, b);
            }
            if (a.positions) a.positions[r] = pos;
            if (a.slots) a.slots[r] = slot;
        }
    }
    // ---- lengths and count, when every CTA has read them ----
    __syncthreads();
    if (tid == 0) {
        int before;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(ticket) : "memory");
        last = before == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    for (int b = tid; b < batch; b += kThreads) {
        const Request q = load_request(a, b);
        a.kv_lens_out[b] = bad ? q.held : q.kept + q.add;
    }
    if (tid == 0) {
        *a.free_count_out = bad ? count : top - n_taken;
        *ticket = 0;                         // ready for the next call
    }
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanArgs &a, StatusBlock *sb, int *ticket, cudaStream_t st)
{
    const int smem = 3 * (int)sizeof(int) * a.batch;
    static std::atomic<int> raised[kMaxDevices];
    const cudaError_t e = raise_smem_limit(kv_plan_kernel, smem, raised);
    if (e != cudaSuccess) return e;
    const int work = a.rows > a.batch ? a.rows : a.batch, sms = device_sms();
    const int ctas = (work + 4 * kThreads - 1) / (4 * kThreads);
    return launch_overlapped(kv_plan_kernel, dim3(ctas < sms ? ctas : sms), dim3(kThreads), smem, st, a, sb, ticket);
}

}  // namespace w4a8
