// Writing the 4-bit key / value cache and reading it back.
//
// Append: a vector (one token, one head, D 16-bit elements) is read once and leaves as D/2 bytes of
// codes and one word: 2 D + D/2 + 4 bytes, so the kernel is bound by memory for prompts and by
// latency for decode steps.  A group of D/8 lanes owns a vector: a lane has eight elements in one
// 16-byte load and writes one code word; the range is reduced over the group by shuffles.  The places
// of a CTA's rows are found once, by a thread each.  Arithmetic was the bound at 182 instructions executed per
// 8 elements of a lane and is no longer at 119 (four vectors quantized together, ranks two to an instruction); hence too the group that
// keeps one row and advances by constants.  Four prompts (611 to 4097 tokens, 8
// heads of 128, 54 MB): 20 us under the profiler, logic pipe 47 % and issue slots 55 % busy; 28.2 us with their read.
// Read is the same walk the other way: 16 sequences (231 MB, 8 heads of 128) 46 us, 5.0 TB/s, issue slots
// 69 % busy.  (A thread per eight elements that found its row by itself took 77 us there.)
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 256;

// Rounded once, values beyond the type's range to its largest finite ones.
template <typename T> __device__ __forceinline__ uint32_t pack2_sat(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2_sat<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(fminf(fmaxf(a, -65504.0f), 65504.0f),
                                        fminf(fmaxf(b, -65504.0f), 65504.0f));
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2_sat<__nv_bfloat16>(float a, float b)
{
    const float m = __uint_as_float(0x7f7f0000u);
    const __nv_bfloat162 h = __floats2bfloat162_rn(fminf(fmaxf(a, -m), m), fminf(fmaxf(b, -m), m));
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Where a row's vectors live: byte offset of its block of head 0, and the token's place in the block.
struct RowPlace {
    long long at;                            // -1: the row reads as zeros; -2: it is left alone
    int s;
};

// Place of one row, found by one thread (a binary search over the row offsets).
__device__ RowPlace place_of(const KvCache &c, const KvBatch &bt, int row, StatusBlock *sb)
{
    int b = row;
    if (bt.cu_rows) {                        // the number of entries 1 .. batch that are <= row
        int lo = 0, hi = bt.batch;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldca(bt.cu_rows + mid) <= row) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
    }
    if (b >= bt.batch) return {-2, 0};       // behind the last sequence
    bool ok;
    const int pos = kv_position_of(bt, b, row, ok);
    if (ok && pos < 0) return {-1, 0};
    const int page = ok ? kv_page_of(c, bt, b, pos) : -1;
    if (page < 0) {
        report_failure(sb, W4A8_ERR_BAD_TABLE, row);
        return {-1, 0};
    }
    const int slot = pos & ((1 << c.page_shift) - 1);
    return {(long long)((size_t)page * c.page_bytes() + (size_t)(slot >> 4) * kv_block_bytes(c.D)), slot & 15};
}

// A group of D/8 lanes owns a row and walks over `vecs` of its 2 * heads vectors (keys of all heads, then values),
// so that its addresses advance by constants; the groups of a CTA own consecutive rows, which are
// neighbours in the cache's blocks.
constexpr int kUnroll = 4;                   // vectors of a group whose loads are in flight together, and that are quantized together

// Sub-range [h0, h1) of the heads that a CTA's vectors v0 .. v0 + nv - 1 cover, for keys (0) or values (1).
__device__ __forceinline__ void heads_of(int v0, int nv, int heads, int value, int &h0, int &h1)
{
    h0 = max(v0 - value * heads, 0);
    h1 = min(v0 + nv - value * heads, heads);
}

// FOUR: kUnroll vectors are quantized together, else one by one.
template <typename T, int D, bool FOUR>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const T *__restrict__ K, const T *__restrict__ V, long long k_stride,
                 long long v_stride, KvCache c, KvBatch bt, int vecs, StatusBlock *sb)
{
    constexpr int LPV = D / 8, GROUPS = kThreads / LPV;
    __shared__ RowPlace place[GROUPS];
    allow_dependents();
    dependent_wait();
    const int group = threadIdx.x / LPV, l = threadIdx.x % LPV;
    const int row0 = blockIdx.x * GROUPS, row = row0 + group, v0 = blockIdx.y * vecs, nv = min(vecs, 2 * c.heads - v0);
    if (threadIdx.x < GROUPS)
        place[threadIdx.x] = row0 + threadIdx.x < bt.rows ? place_of(c, bt, row0 + threadIdx.x, sb) : RowPlace{-2, 0};
    __syncthreads();
    const RowPlace p = place[group];
    const size_t head_bytes = ((size_t)1 << c.page_shift) * (D + 8);
    const bool here = p.at >= 0;
#pragma unroll
    for (int value = 0; value < 2; ++value) {
        int h0, h1;
        heads_of(v0, nv, c.heads, value, h0, h1);
        const T *from = (value ? V + row * v_stride : K + row * k_stride) + (size_t)h0 * D + 8 * l;
        uint8_t *to = c.pages + p.at + h0 * head_bytes;
        const int code_at = kv_code_offset(D, value, p.s, l), word_at = kv_word_offset(D, value, p.s);
        // (lanes without a row take part in the shuffles)
        for (int h = h0; h < h1; h += kUnroll) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                raw[j] = make_uint4(0u, 0u, 0u, 0u);
                if (here && h + j < h1) raw[j] = __ldcs(reinterpret_cast<const uint4 *>(from + j * D));
            }
            float x[kUnroll][8], lo[kUnroll], hi[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                if (!FOUR && h + j >= h1) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 f = to_float2<T>((&raw[j].x)[k]);
                    x[j][2 * k] = f.x;
                    x[j][2 * k + 1] = f.y;
                }
                lo[j] = hi[j] = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    lo[j] = min3(lo[j], x[j][k], x[j][k + 1]);
                    hi[j] = max3(hi[j], x[j][k], x[j][k + 1]);
                }
                if constexpr (!FOUR) {
#pragma unroll
                    for (int o = LPV / 2; o > 0; o >>= 1) {
                        lo[j] = fminf(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], o));
                        hi[j] = fmaxf(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], o));
                    }
                    float r;
                    int z;
                    const uint32_t word = kv_range_word(lo[j], hi[j], r, z), codes = kv_code_word(x[j], r, kv_twice(z));
                    if (here) {
                        *reinterpret_cast<uint32_t *>(to + j * head_bytes + code_at) = codes;
                        if (l == 0) *reinterpret_cast<uint32_t *>(to + j * head_bytes + word_at) = word;
                    }
                }
            }
            if constexpr (FOUR) {
                float my_r;
                int my_z;
                const uint32_t my_word = kv_four_words<LPV>(lo, hi, l, my_r, my_z), my_zz = kv_twice(my_z);
                constexpr int OWN = LPV / kUnroll;           // the words, by one lane each
                const int mine = (l / OWN & 1) + (l / OWN & 2);
                if (l % OWN == 0 && here && h + mine < h1) *reinterpret_cast<uint32_t *>(to + mine * head_bytes + word_at) = my_word;
#pragma unroll
                for (int j = 0; j < kUnroll; ++j) {
                    const uint32_t zz = __shfl_sync(0xffffffffu, my_zz, kv_owner_of<LPV>(j), LPV);
                    const float r = __shfl_sync(0xffffffffu, my_r, kv_owner_of<LPV>(j), LPV);
                    if (here && h + j < h1) *reinterpret_cast<uint32_t *>(to + j * head_bytes + code_at) = kv_code_word(x[j], r, zz);
                }
            }
            from += kUnroll * D;
            to += kUnroll * head_bytes;
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(KvCache c, KvBatch bt, T *__restrict__ K, T *__restrict__ V, int vecs, StatusBlock *sb)
{
    constexpr int LPV = D / 8, GROUPS = kThreads / LPV;
    __shared__ RowPlace place[GROUPS];
    allow_dependents();
    dependent_wait();
    const int group = threadIdx.x / LPV, l = threadIdx.x % LPV;
    const int row0 = blockIdx.x * GROUPS, row = row0 + group, v0 = blockIdx.y * vecs, nv = min(vecs, 2 * c.heads - v0);
    if (threadIdx.x < GROUPS)
        place[threadIdx.x] = row0 + threadIdx.x < bt.rows ? place_of(c, bt, row0 + threadIdx.x, sb) : RowPlace{-2, 0};
    __syncthreads();
    const RowPlace p = place[group];
    if (p.at == -2) return;                  // no row, or one behind the last sequence
    const size_t head_bytes = ((size_t)1 << c.page_shift) * (D + 8);
#pragma unroll
    for (int value = 0; value < 2; ++value) {
        int h0, h1;
        heads_of(v0, nv, c.heads, value, h0, h1);
        T *to = (value ? V : K) + ((size_t)row * c.heads + h0) * D + 8 * l;
        const uint8_t *from = c.pages + (p.at < 0 ? 0 : p.at) + h0 * head_bytes;
        const int code_at = kv_code_offset(D, value, p.s, l), word_at = kv_word_offset(D, value, p.s);
        for (int h = h0; h < h1; h += kUnroll) {
            uint32_t codes[kUnroll], word[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                codes[j] = word[j] = 0u;     // an absent vector: step 0
                if (p.at >= 0 && h + j < h1) {
                    codes[j] = __ldca(reinterpret_cast<const uint32_t *>(from + j * head_bytes + code_at));
                    word[j] = __ldca(reinterpret_cast<const uint32_t *>(from + j * head_bytes + word_at));
                }
            }
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                if (h + j >= h1) break;
                const float step = 2.0f * __uint_as_float(word[j] & ~15u);       // (a step is below 2^126)
                __half2 o[4];
                kv_levels(codes[j], (int)(word[j] & 15u), o);
                float2 f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = __half22float2(o[k]);
                const uint4 out = {pack2_sat<T>(__fmul_rn(f[0].x, step), __fmul_rn(f[1].x, step)),
                                   pack2_sat<T>(__fmul_rn(f[2].x, step), __fmul_rn(f[3].x, step)),
                                   pack2_sat<T>(__fmul_rn(f[0].y, step), __fmul_rn(f[1].y, step)),
                                   pack2_sat<T>(__fmul_rn(f[2].y, step), __fmul_rn(f[3].y, step))};
                __stcs(reinterpret_cast<uint4 *>(to + j * D), out);
            }
            to += kUnroll * D;
            from += kUnroll * head_bytes;
        }
    }
}

// Vectors per CTA: all of a row's where the rows alone give eight CTAs per SM, fewer (down to one) else.
struct Shape {
    dim3 grid;
    int vecs;
};
Shape shape_of(int D, int heads, int rows)
{
    const int groups = kThreads / (D / 8), across = (rows + groups - 1) / groups;
    const int parts = (8 * device_sms() + across - 1) / across;
    Shape s;
    s.vecs = parts >= 2 * heads ? 1 : (2 * heads + parts - 1) / parts;
    s.grid = dim3(across, (2 * heads + s.vecs - 1) / s.vecs);
    return s;
}

template <typename T, int D>
cudaError_t append(const void *K, const void *V, long long ks, long long vs, const KvCache &c,
                   const KvBatch &bt, StatusBlock *sb, cudaStream_t st)
{
    Shape s = shape_of(D, c.heads, bt.rows);
    const T *k = static_cast<const T *>(K), *v = static_cast<const T *>(V);
    // (four at a time where a CTA has as many of a row: 10348 rows of 8 heads 17.4 us, one by one 19.0; 128 rows, a vector or two a row: 3.4 us
    // four at a time, 2.9 one by one)
    if (s.vecs < kUnroll || c.heads < kUnroll)
        return launch_overlapped(kv_append_kernel<T, D, false>, s.grid, dim3(kThreads), 0, st, k, v, ks, vs, c, bt, s.vecs, sb);
    s.vecs = (s.vecs + kUnroll - 1) / kUnroll * kUnroll;
    s.grid.y = (2 * c.heads + s.vecs - 1) / s.vecs;
    return launch_overlapped(kv_append_kernel<T, D, true>, s.grid, dim3(kThreads), 0, st, k, v, ks, vs, c, bt, s.vecs, sb);
}
template <typename T, int D>
cudaError_t read(const KvCache &c, const KvBatch &bt, void *K, void *V, StatusBlock *sb,
                 cudaStream_t st)
{
    const Shape s = shape_of(D, c.heads, bt.rows);
    return launch_overlapped(kv_read_kernel<T, D>, s.grid, dim3(kThreads), 0, st, c, bt,
                             static_cast<T *>(K), static_cast<T *>(V), s.vecs, sb);
}

}  // namespace

cudaError_t launch_kv_append(const void *K, const void *V, int bf16, long long k_stride,
                             long long v_stride, const KvCache &c, const KvBatch &bt,
                             StatusBlock *sb, cudaStream_t st)
{
    if (c.D == 64)
        return bf16 ? append<__nv_bfloat16, 64>(K, V, k_stride, v_stride, c, bt, sb, st)
                    : append<__half, 64>(K, V, k_stride, v_stride, c, bt, sb, st);
    return bf16 ? append<__nv_bfloat16, 128>(K, V, k_stride, v_stride, c, bt, sb, st)
                : append<__half, 128>(K, V, k_stride, v_stride, c, bt, sb, st);
}

cudaError_t launch_kv_read(const KvCache &c, const KvBatch &bt, void *K, void *V, int bf16,
                           StatusBlock *sb, cudaStream_t st)
{
    if (c.D == 64)
        return bf16 ? read<__nv_bfloat16, 64>(c, bt, K, V, sb, st) : read<__half, 64>(c, bt, K, V, sb, st);
    return bf16 ? read<__nv_bfloat16, 128>(c, bt, K, V, sb, st) : read<__half, 128>(c, bt, K, V, sb, st);
}

}  // namespace w4a8
