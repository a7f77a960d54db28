// Attention over the 4-bit cache: one CTA per row and query head, one pass over the keys with the
// running maximum and sum of the softmax, everything in binary32 on the CUDA cores.
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 128;

__device__ __forceinline__ float load16(const void *p, size_t i, int bf16)
{
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i])
                : __half2float(static_cast<const __half *>(p)[i]);
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv_attention_kernel(KvAttnArgs a, StatusBlock *sb)
{
    __shared__ float q[D], p[kThreads], red[kThreads / 32], vstep[kThreads];
    allow_dependents();
    dependent_wait();
    const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
    const KvBatch &bt = a.batch;
    const int b = kv_sequence_of(bt, row);
    if (b >= bt.batch) return;
    bool ok;
    const int pos = kv_position_of(bt, b, row, ok);
    if (!ok && tid == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
    const int hi = !ok || pos < 0 ? 0 : (a.causal ? pos + 1 : __ldg(bt.kv_lens + b));
    const int lo = a.window > 0 ? max(0, pos + 1 - a.window) : 0;
    for (int d = tid; d < D; d += kThreads)
        q[d] = load16(a.Q, (size_t)(row * a.q_stride) + (size_t)head * D + d, a.q_bf16);
    __syncthreads();
    const int kvh = head / (a.q_heads / a.cache.heads);
    float m = -INFINITY, sum = 0.0f, acc = 0.0f;
    const float scale = a.scale;
    for (int base = lo & ~15; base < hi; base += kThreads) {
        const int j = base + tid;
        float sc = -INFINITY;
        const uint8_t *blk = nullptr;
        if (j >= lo && j < hi) {
            const int page = kv_page_of(a.cache, bt, b, j);
            if (page < 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
            else blk = kv_block_at(a.cache, page, kvh, j & ((1 << a.cache.page_shift) - 1));
        }
        vstep[tid] = 0.0f;
        if (blk) {
            const uint32_t wk = *reinterpret_cast<const uint32_t *>(blk + kv_word_offset(D, 0, j & 15));
            float dot = 0.0f;
            for (int w = 0; w < D / 8; ++w) {
                const uint32_t c = *reinterpret_cast<const uint32_t *>(blk + kv_code_offset(D, 0, j & 15, w));
                for (int e = 0; e < 8; ++e)
                    dot = fmaf(q[8 * w + e], kv_level(kv_rank_at(c, e), (int)(wk & 15u)), dot);
            }
            sc = dot * __uint_as_float(wk & ~15u) * scale;
        }
        float mx = sc;
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if ((tid & 31) == 0) red[tid >> 5] = mx;
        __syncthreads();
        mx = m;
        for (int w = 0; w < kThreads / 32; ++w) mx = fmaxf(mx, red[w]);
        const float keep = mx == -INFINITY ? 1.0f : expf(m - mx);
        m = mx;
        p[tid] = sc == -INFINITY ? 0.0f : expf(sc - m);
        __syncthreads();
        sum *= keep;
        acc *= keep;
        const int n = min(kThreads, hi - base);
        for (int i = 0; i < n; ++i) {
            sum += p[i];
            const int j2 = base + i;
            if (tid < D && p[i] != 0.0f) {
                const int page = kv_page_of(a.cache, bt, b, j2);
                const uint8_t *bl = kv_block_at(a.cache, page, kvh, j2 & ((1 << a.cache.page_shift) - 1));
                const uint32_t wv = *reinterpret_cast<const uint32_t *>(bl + kv_word_offset(D, 1, j2 & 15));
                const uint32_t c = *reinterpret_cast<const uint32_t *>(bl + kv_code_offset(D, 1, j2 & 15, tid >> 3));
                acc = fmaf(p[i], kv_level(kv_rank_at(c, tid & 7), (int)(wv & 15u)) * __uint_as_float(wv & ~15u), acc);
            }
        }
        __syncthreads();
    }
    const size_t at = (size_t)row * a.q_heads + head;
    if (tid < D) {
        const float o = sum > 0.0f ? acc / sum : 0.0f;
        if (a.o_bf16) static_cast<__nv_bfloat16 *>(a.O)[at * D + tid] = __float2bfloat16_rn(o);
        else static_cast<__half *>(a.O)[at * D + tid] = __float2half_rn(fminf(fmaxf(o, -65504.0f), 65504.0f));
    }
    if (a.lse && tid == 0) a.lse[at] = sum > 0.0f ? m + logf(sum) : -INFINITY;
}

}  // namespace

size_t kv_attention_workspace(int, int, int, int, int) { return sizeof(StatusBlock); }

cudaError_t launch_kv_attention(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st)
{
    StatusBlock *sb = reinterpret_cast<StatusBlock *>(workspace);
    const dim3 grid(a.batch.rows, a.q_heads);
    return a.cache.D == 64 ? launch_overlapped(kv_attention_kernel<64>, grid, dim3(kThreads), 0, st, a, sb)
                           : launch_overlapped(kv_attention_kernel<128>, grid, dim3(kThreads), 0, st, a, sb);
}

}  // namespace w4a8
