// Accepted drafted tokens move to the front of the drafted ones: slot base + i takes the keys and values of slot
// base + path[i], base = the sequence's tokens without the call's rows.
//
// A moved vector is D/2 bytes of codes and a word, copied as they are.  A group of D/8 lanes owns one vector (a head's key or value) of a
// sequence and walks along its path, so that every byte is read and written by the same lane; in an ascending path path[i] >= i (a place
// that is not is left out, negative ones among them), so the slot that the i-th copy fills is the source of no later copy: the copies need
// no order among lanes, and a lane may load several in front of its first store.  Few bytes move: the time is a launch and four dependent accesses (lengths with
// the path, page table, source, destination).  Eight sequences of 8 heads 2.9 us, 64 of 32 heads with up to nine accepted rows 5.1 us (5 MB).
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 128;                  // copies whose places a CTA looks up at a time
constexpr int kUnroll = 4;                   // copies of a lane whose loads are in flight together

// Where token pos of sequence b lies: byte offset of its block of head 0, and the token's place in the block.
struct Slot {
    long long at;                            // -1: nowhere
    int s;
};
__device__ __forceinline__ Slot slot_of(const KvCache &c, const KvBatch &bt, int b, int pos)
{
    const int page = kv_page_of(c, bt, b, pos);
    if (page < 0) return {-1, 0};
    const int place = pos & ((1 << c.page_shift) - 1);
    return {(long long)((size_t)page * c.page_bytes() + (size_t)(place >> 4) * kv_block_bytes(c.D)), place & 15};
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv_accept_kernel(const KvCache c, const KvBatch bt, const KvPaths paths, StatusBlock *sb)
{
    constexpr int LPV = D / 8, GROUPS = kThreads / LPV;
    __shared__ Slot from[kBatch], to[kBatch];
    allow_dependents();
    dependent_wait();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int32_t *path = paths.accepted + (size_t)b * paths.most;
    // (the first places travel with the lengths)
    const int first = tid < min(kBatch, paths.most) ? __ldca(path + tid) : 0;
    const int len = __ldca(bt.kv_lens + b);
    const int row0 = bt.cu_rows ? __ldca(bt.cu_rows + b) : b, row1 = bt.cu_rows ? __ldca(bt.cu_rows + b + 1) : b + 1;
    int count = __ldca(paths.accept_lens + b);
    const int kept = paths.kept ? __ldca(paths.kept + b) : 0;
    const int n = row1 - row0, base = len - n;
    const bool good = row0 >= 0 && n >= 0 && row1 <= bt.rows && base >= 0 && (long long)len <= (long long)bt.max_pages << c.page_shift && count >= 0 &&
                      count <= paths.most && count <= n;
    if (!good) {
        if (tid == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, b);
        count = 0;
    }
    // (a plan that was refused gives no sequence rows, and as their lengths those that the pages were taken for)
    if (paths.kv_lens_out && blockIdx.y == 0 && tid == 0) paths.kv_lens_out[b] = paths.kept && (n == 0 || !good) ? kept : max(base, 0) + count;
    const size_t head_bytes = ((size_t)1 << c.page_shift) * (D + 8);
    const int l = tid % LPV, vec = blockIdx.y * GROUPS + tid / LPV;
    const int head = vec >> 1, value = vec & 1;
    uint8_t *pages = c.pages + head * head_bytes;
    for (int i0 = 0; i0 < count; i0 += kBatch) {
        const int here = min(kBatch, count - i0);
        if (i0) __syncthreads();             // the places of the copies before are no longer needed
        for (int k = tid; k < here; k += kThreads) {
            const int i = i0 + k, j = i0 ? __ldca(path + i) : first, before = i ? __ldca(path + i - 1) : -1;
            Slot x = {-1, 0}, y = {-1, 0};
            if (j < i || j <= before || j >= n) report_failure(sb, W4A8_ERR_BAD_TABLE, b);
            else if (j != i) {
                x = slot_of(c, bt, b, base + j);
                y = slot_of(c, bt, b, base + i);
                if (x.at < 0 || y.at < 0) {
                    report_failure(sb, W4A8_ERR_BAD_TABLE, b);
                    x.at = -1;
                }
            }
            from[k] = x;
            to[k] = y;
        }
        __syncthreads();
        if (head >= c.heads) continue;
        for (int k = 0; k < here; k += kUnroll) {
            uint32_t codes[kUnroll], word[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                codes[u] = word[u] = 0u;
                if (k + u >= here || from[k + u].at < 0) continue;
                const uint8_t *p = pages + from[k + u].at;
                codes[u] = __ldca(reinterpret_cast<const uint32_t *>(p + kv_code_offset(D, value, from[k + u].s, l)));
                if (l == 0) word[u] = __ldca(reinterpret_cast<const uint32_t *>(p + kv_word_offset(D, value, from[k + u].s)));
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (k + u >= here || from[k + u].at < 0) continue;
                uint8_t *p = pages + to[k + u].at;
                *reinterpret_cast<uint32_t *>(p + kv_code_offset(D, value, to[k + u].s, l)) = codes[u];
                if (l == 0) *reinterpret_cast<uint32_t *>(p + kv_word_offset(D, value, to[k + u].s)) = word[u];
            }
        }
    }
}

}  // namespace

cudaError_t launch_kv_accept(const KvCache &c, const KvBatch &bt, const KvPaths &paths, StatusBlock *sb, cudaStream_t st)
{
    const int groups = kThreads / (c.D / 8);
    const dim3 grid(bt.batch, (2 * c.heads + groups - 1) / groups);
    return c.D == 64 ? launch_overlapped(kv_accept_kernel<64>, grid, dim3(kThreads), 0, st, c, bt, paths, sb)
                     : launch_overlapped(kv_accept_kernel<128>, grid, dim3(kThreads), 0, st, c, bt, paths, sb);
}

}  // namespace w4a8
