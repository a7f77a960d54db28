// Writing the 4-bit key / value cache and reading it back.
//
// Append: a vector (one token, one head, D 16-bit elements) is read once and leaves as D/2 bytes of
// codes and one word: 2 D + D/2 + 4 bytes, so the kernel is bound by memory for prompts and by
// latency for decode steps.  A group of D/8 lanes owns a vector: a lane has eight elements in one
// 16-byte load and writes one code word; the range is reduced over the group by shuffles.  A warp
// takes kVecs groups of vectors of one row at once, all loads issued before the first is used.
// Read is the same walk the other way.
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 128;

template <typename T> __device__ __forceinline__ float2 to_float2(uint32_t v);
template <> __device__ __forceinline__ float2 to_float2<__half>(uint32_t v)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}
template <> __device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

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

// D: head dimension.  VECS: vectors per lane group.
template <typename T, int D, int VECS>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const T *__restrict__ K, const T *__restrict__ V, long long k_stride,
                 long long v_stride, KvCache c, KvBatch bt, int units_per_row, StatusBlock *sb)
{
    allow_dependents();
    dependent_wait();
    constexpr int LPV = D / 8, VPW = 32 / LPV;
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const long long row64 = unit / units_per_row;
    if (row64 >= bt.rows) return;
    const int row = (int)row64, part = (int)(unit - row64 * units_per_row);
    const int l = lane % LPV, first = part * (VPW * VECS) + lane / LPV;
    const int nvec = 2 * c.heads;            // keys of all heads, then values
    uint4 raw[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int v = first + i * VPW;
        raw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (v < nvec) {
            const T *p = v < c.heads ? K + row * k_stride + (size_t)v * D
                                     : V + row * v_stride + (size_t)(v - c.heads) * D;
            raw[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + l);
        }
    }
    const int b = kv_sequence_of(bt, row);
    if (b >= bt.batch) return;               // behind the last sequence
    bool ok;
    const int pos = kv_position_of(bt, b, row, ok);
    const int page = ok && pos >= 0 ? kv_page_of(c, bt, b, pos) : -1;
    if (page < 0) {
        if ((!ok || pos >= 0) && lane == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
        return;
    }
    const int slot = pos & ((1 << c.page_shift) - 1), s = slot & 15;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int v = first + i * VPW;
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = to_float2<T>((&raw[i].x)[j]);
            x[2 * j] = f.x;
            x[2 * j + 1] = f.y;
        }
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fminf(lo, x[j]);
            hi = fmaxf(hi, x[j]);
        }
#pragma unroll
        for (int o = LPV / 2; o > 0; o >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        float r;
        int z;
        const uint32_t word = kv_range_word(lo, hi, r, z);
        uint32_t k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] = kv_rank(x[j], r, z);
        const uint32_t codes = kv_half(k[0], k[1], k[2], k[3]) | (kv_half(k[4], k[5], k[6], k[7]) << 16);
        if (v < nvec) {
            const int val = v >= c.heads;
            uint8_t *blk = kv_block_at(c, page, val ? v - c.heads : v, slot);
            *reinterpret_cast<uint32_t *>(blk + kv_code_offset(D, val, s, l)) = codes;
            if (l == 0) *reinterpret_cast<uint32_t *>(blk + kv_word_offset(D, val, s)) = word;
        }
    }
}

template <typename T, int D, int VECS>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(KvCache c, KvBatch bt, T *__restrict__ K, T *__restrict__ V, int units_per_row,
               StatusBlock *sb)
{
    allow_dependents();
    dependent_wait();
    constexpr int LPV = D / 8, VPW = 32 / LPV;
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const long long row64 = unit / units_per_row;
    if (row64 >= bt.rows) return;
    const int row = (int)row64, part = (int)(unit - row64 * units_per_row);
    const int l = lane % LPV, first = part * (VPW * VECS) + lane / LPV;
    const int nvec = 2 * c.heads;
    const int b = kv_sequence_of(bt, row);
    if (b >= bt.batch) return;
    bool ok;
    const int pos = kv_position_of(bt, b, row, ok);
    const int page = ok && pos >= 0 ? kv_page_of(c, bt, b, pos) : -1;
    if (page < 0 && (!ok || pos >= 0) && lane == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
    const int slot = pos & ((1 << c.page_shift) - 1), s = slot & 15;
    uint32_t codes[VECS], word[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int v = first + i * VPW;
        codes[i] = word[i] = 0u;             // an absent vector: step 0
        if (v < nvec && page >= 0) {
            const int val = v >= c.heads;
            const uint8_t *blk = kv_block_at(c, page, val ? v - c.heads : v, slot);
            codes[i] = *reinterpret_cast<const uint32_t *>(blk + kv_code_offset(D, val, s, l));
            word[i] = *reinterpret_cast<const uint32_t *>(blk + kv_word_offset(D, val, s));
        }
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int v = first + i * VPW;
        if (v >= nvec) continue;
        const float step = __uint_as_float(word[i] & ~15u);
        const int z = (int)(word[i] & 15u);
        uint4 out;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = __fmul_rn(kv_level(kv_rank_at(codes[i], 2 * j), z), step);
            const float d = __fmul_rn(kv_level(kv_rank_at(codes[i], 2 * j + 1), z), step);
            (&out.x)[j] = pack2_sat<T>(a, d);
        }
        T *p = v < c.heads ? K + ((size_t)row * c.heads + v) * D
                           : V + ((size_t)row * c.heads + v - c.heads) * D;
        __stcs(reinterpret_cast<uint4 *>(p) + l, out);
    }
}

// Units (warps) per row and CTAs for `vecs` vectors per lane group.
struct Grid {
    int per_row;
    unsigned ctas;
};
Grid grid_of(int D, int heads, int rows, int vecs)
{
    const int per_warp = 32 / (D / 8) * vecs;
    Grid g;
    g.per_row = (2 * heads + per_warp - 1) / per_warp;
    g.ctas = (unsigned)(((long long)g.per_row * rows + kThreads / 32 - 1) / (kThreads / 32));
    return g;
}

template <typename T, int D>
cudaError_t append(const void *K, const void *V, long long ks, long long vs, const KvCache &c,
                   const KvBatch &bt, StatusBlock *sb, cudaStream_t st)
{
    const Grid g = grid_of(D, c.heads, bt.rows, 4);
    return launch_overlapped(kv_append_kernel<T, D, 4>, dim3(g.ctas), dim3(kThreads), 0, st,
                             static_cast<const T *>(K), static_cast<const T *>(V), ks, vs, c, bt,
                             g.per_row, sb);
}
template <typename T, int D>
cudaError_t read(const KvCache &c, const KvBatch &bt, void *K, void *V, StatusBlock *sb,
                 cudaStream_t st)
{
    const Grid g = grid_of(D, c.heads, bt.rows, 4);
    return launch_overlapped(kv_read_kernel<T, D, 4>, dim3(g.ctas), dim3(kThreads), 0, st, c, bt,
                             static_cast<T *>(K), static_cast<T *>(V), g.per_row, sb);
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
