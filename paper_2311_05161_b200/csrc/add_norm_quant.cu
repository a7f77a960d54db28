// Residual addition, normalisation and token-wise INT8 quantizer in one pass.
//
// Between two sub-blocks of a decoder layer the branch's output joins the residual stream and the
// normalised stream becomes the next linear's INT8 input.  One launch reads the branch and the
// stream once and writes the stream and the codes: 7 bytes per element with a 16-bit stream, 11
// with a 32-bit one, where addition and w4a8_norm_quantize_act apart move 9 (13).
//
// A thread keeps vectors of eight of a token's elements in registers through all phases (load, sum, maximum, codes:
// two or three dependent steps across the CTA).  Bound by memory for prompts, as far as enough tokens are in
// flight per SM to cover those steps; three forms (measured on B200, against 6.54 TB/s of a copy):
//  - several tokens per CTA, weights in registers, the next two tokens on their way into shared memory:
//    4000 tokens of 5120, RMS, bfloat16: 32.3 us, 4.4 TB/s (37.4 us without); 2048 of 4096: 14.0 us (15.9);
//  - few tokens: one per CTA, sixteen elements per thread: one token of 4096 2.7 us, the launch and three
//    steps of latency;
//  - many long tokens: one per CTA, 32 elements per thread (fewer threads, so more tokens fit an SM): 2048 of
//    9216, LayerNorm, binary32 stream: 41.9 us, 5.0 TB/s (46.7 with sixteen).
//
// The sums are binary64 from the elements on: their order then does not matter to the binary32
// values that are rounded from them (but for one case in about 2^28), so any other implementation in
// binary64 gives the same codes.
#include <atomic>

#include "common.cuh"
#include "quant_math.cuh"

namespace w4a8 {

namespace {

// Sixteen bytes from global memory that are read once, or from shared memory.
template <bool STREAM> __device__ __forceinline__ uint4 fetch(const void *p)
{
    return STREAM ? __ldcs(static_cast<const uint4 *>(p)) : *static_cast<const uint4 *>(p);
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// Eight elements as binary32.
template <typename T> struct Vec8;
template <> struct Vec8<__half> {
    template <bool STREAM = true> static __device__ __forceinline__ void load(const __half *p, float (&x)[8])
    {
        const uint4 v = fetch<STREAM>(p);
        scaled8(v, nullptr, 0, x);
    }
    static __device__ __forceinline__ void round_store(__half *p, float (&x)[8])
    {
        uint4 v;
        __half2 *h = reinterpret_cast<__half2 *>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            const float2 f = __half22float2(h[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
        *reinterpret_cast<uint4 *>(p) = v;
    }
};
template <> struct Vec8<__nv_bfloat16> {
    template <bool STREAM = true> static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&x)[8])
    {
        const uint4 v = fetch<STREAM>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float((&v.x)[i] << 16);
            x[2 * i + 1] = __uint_as_float((&v.x)[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void round_store(__nv_bfloat16 *p, float (&x)[8])
    {
        uint4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            (&v.x)[i] = *reinterpret_cast<const uint32_t *>(&h);
            x[2 * i] = __uint_as_float((&v.x)[i] << 16);
            x[2 * i + 1] = __uint_as_float((&v.x)[i] & 0xffff0000u);
        }
        *reinterpret_cast<uint4 *>(p) = v;
    }
};
template <> struct Vec8<float> {
    template <bool STREAM = true> static __device__ __forceinline__ void load(const float *p, float (&x)[8])
    {
        const uint4 v[2] = {fetch<STREAM>(p), fetch<STREAM>(p + 4)};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((&v[i >> 2].x)[i & 3]);
    }
    static __device__ __forceinline__ void round_store(float *p, float (&x)[8])
    {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};

// |x| as binary64 by integer instructions: the conversion instruction issues at a sixteenth of their rate and
// bounded the kernel.  Zero and subnormal numbers come out near 2^-127, which no square sum with a positive
// eps beside it can tell from zero.
__device__ __forceinline__ double magnitude(float x)
{
    const uint32_t b = __float_as_uint(x);
    return __hiloint2double((int)((b << 1 >> 4) + 0x38000000u), (int)(b << 29));
}

__device__ __forceinline__ double cta_sum(double v, double *buf, int lane, int warp, int nwarps)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (nwarps == 1) return v;
    if (lane == 0) buf[warp] = v;
    __syncthreads();
    v = buf[0];
    for (int w = 1; w < nwarps; ++w) v += buf[w];
    return v;
}

constexpr int kAhead = 2;                    // tokens on their way per CTA in the pipelined form

// EV vectors of eight elements per thread.  PIPE: the CTA walks over tokens with its weights in registers; every
// thread copies its own elements of the next kAhead tokens into shared memory in the background (nobody
// else reads them, so no barrier is involved).
template <typename TX, typename TR, bool LAYER, int EV, bool PIPE>
__global__ void __launch_bounds__(EV == 2 && !PIPE ? 1024 : 512, PIPE ? 2 : 1)
add_norm_quant_kernel(const TX *__restrict__ X, const TR *residual, TR *residual_out,
                      const float *__restrict__ weight, const float *__restrict__ bias, float eps,
                      double inv_k, int M, int K, int8_t *__restrict__ Xq, float *__restrict__ tok_scale)
{
    __shared__ double red_mean[2][32], red_sq[2][32];
    __shared__ float red_max[2][32];
    extern __shared__ __align__(16) uint8_t ahead[];
    allow_dependents();
    dependent_wait();
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 31, warp = tid >> 5, nwarps = T >> 5;
    const int nvec = K >> 3;
    const size_t stage_bytes = (size_t)EV * T * 8 * (sizeof(TX) + sizeof(TR));
    auto prefetch = [&](int m, int stage) {
        if (m < M) {
#pragma unroll
            for (int i = 0; i < EV; ++i) {
                const int v = tid + i * T;
                if (v >= nvec) continue;
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(ahead + stage * stage_bytes);
                copy16(to + v * 8 * sizeof(TX), X + (size_t)m * K + v * 8);
#pragma unroll
                for (int p = 0; p < (int)sizeof(TR) / 2; ++p)
                    copy16(to + EV * T * 8 * sizeof(TX) + v * 8 * sizeof(TR) + 16 * p,
                           reinterpret_cast<const uint8_t *>(residual + (size_t)m * K + v * 8) + 16 * p);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // with few elements per thread there are registers for the weights too, on their way during the sums
    float4 wa[EV], wb[EV];
    if (EV == 2) {
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const int v = tid + i * T;
            if (v < nvec) {
                wa[i] = __ldca(reinterpret_cast<const float4 *>(weight) + 2 * v);
                wb[i] = __ldca(reinterpret_cast<const float4 *>(weight) + 2 * v + 1);
            }
        }
    }
    if (PIPE) {
#pragma unroll
        for (int s = 0; s < kAhead; ++s) prefetch(blockIdx.x + s * gridDim.x, s);
    }
    int turn = 0, stage = 0;
    for (int m = blockIdx.x; m < M; m += gridDim.x, turn ^= 1) {
        const size_t row = (size_t)m * K;
        float x[EV][8], y[EV][8];
        if (PIPE) asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const int v = tid + i * T;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.0f;
            if (v < nvec) {
                if (PIPE) {
                    const uint8_t *from = ahead + stage * stage_bytes;
                    Vec8<TX>::template load<false>(reinterpret_cast<const TX *>(from) + v * 8, y[i]);
                    Vec8<TR>::template load<false>(reinterpret_cast<const TR *>(from + EV * T * 8 * sizeof(TX)) + v * 8, x[i]);
                } else {
                    Vec8<TX>::load(X + row + v * 8, y[i]);
                    Vec8<TR>::load(residual + row + v * 8, x[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const int v = tid + i * T;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = __fadd_rn(x[i][e], y[i][e]);
            if (v < nvec) Vec8<TR>::round_store(residual_out + row + v * 8, x[i]);
        }
        if (PIPE) {
            prefetch(m + kAhead * gridDim.x, stage);
            stage = stage + 1 == kAhead ? 0 : stage + 1;
        }
        if (LAYER) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < EV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += (double)x[i][e];
            const float mu = __double2float_rn(cta_sum(s, red_mean[turn], lane, warp, nwarps) * inv_k);
#pragma unroll
            for (int i = 0; i < EV; ++i)
                if (tid + i * T < nvec)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[i][e] = __fsub_rn(x[i][e], mu);
        }
        double sq = 0.0;
#pragma unroll
        for (int i = 0; i < EV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = magnitude(x[i][e]);
                sq = fma(d, d, sq);
            }
        sq = cta_sum(sq, red_sq[turn], lane, warp, nwarps);
        const float r = __double2float_rn(rsqrt(sq * inv_k + (double)eps));
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const int v = tid + i * T;
            if (v < nvec) {
                if (EV != 2) {
                    wa[i] = __ldca(reinterpret_cast<const float4 *>(weight) + 2 * v);
                    wb[i] = __ldca(reinterpret_cast<const float4 *>(weight) + 2 * v + 1);
                }
                const float w[8] = {wa[i].x, wa[i].y, wa[i].z, wa[i].w, wb[i].x, wb[i].y, wb[i].z, wb[i].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = __fmul_rn(__fmul_rn(x[i][e], r), w[e]);
                if (bias) {
                    const float4 ba = __ldca(reinterpret_cast<const float4 *>(bias) + 2 * v);
                    const float4 bb = __ldca(reinterpret_cast<const float4 *>(bias) + 2 * v + 1);
                    const float b[8] = {ba.x, ba.y, ba.z, ba.w, bb.x, bb.y, bb.z, bb.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[i][e] = __fadd_rn(x[i][e], b[e]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[i][e]));
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        if (nwarps > 1) {
            float *buf = red_max[turn];        // (two sets in turn: a fast warp may be one token ahead)
            if (lane == 0) buf[warp] = amax;
            __syncthreads();
            amax = buf[0];
            for (int w = 1; w < nwarps; ++w) amax = fmaxf(amax, buf[w]);
        }
        const float q = amax > 0.0f ? __fdiv_rn(127.0f, amax) : 0.0f;
        if (tid == 0) tok_scale[m] = __fdiv_rn(amax, 127.0f);
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const int v = tid + i * T;
            if (v < nvec) *reinterpret_cast<uint2 *>(Xq + row + v * 8) = quantize8(x[i], q);
        }
        if (!PIPE) break;                  // one token per CTA
    }
}

template <typename TX, typename TR, bool LAYER>
cudaError_t launch(const void *X, const void *residual, void *residual_out, const float *weight,
                   const float *bias, float eps, int M, int K, int8_t *Xq, float *tok_scale,
                   cudaStream_t st)
{
    auto threads_of = [&](int ev) { return ((K / 8 + ev - 1) / ev + 31) / 32 * 32; };
    auto with = [&](auto kernel, int ctas, int threads, size_t smem) {
        return launch_overlapped(kernel, dim3(ctas), dim3(threads), smem, st, static_cast<const TX *>(X),
                                 static_cast<const TR *>(residual), static_cast<TR *>(residual_out), weight, bias, eps,
                                 1.0 / K, M, K, Xq, tok_scale);
    };
    const int threads = threads_of(2), sms = device_sms();
    if (M > 2 * sms && threads <= 512) {
        // several tokens per CTA: as many CTAs as stay resident (64 registers per thread, kAhead tokens in shared memory)
        const size_t smem = (size_t)kAhead * 2 * threads * 8 * (sizeof(TX) + sizeof(TR));
        int per_sm = 1024 / threads;
        if (per_sm > (int)(216 * 1024 / (smem + 2560))) per_sm = (int)(216 * 1024 / (smem + 2560));
        if (per_sm > 16) per_sm = 16;
        if (per_sm >= 2) {
            auto kernel = add_norm_quant_kernel<TX, TR, LAYER, 2, true>;
            static std::atomic<int> raised[kMaxDevices];
            const cudaError_t e = raise_smem_limit(kernel, (int)smem, raised);
            if (e != cudaSuccess) return e;
            return with(kernel, M < per_sm * sms ? M : per_sm * sms, threads, smem);
        }
    }
    // Few tokens: more threads, fewer steps each.  Many long ones: fewer threads keep more of them in flight per SM.
    return M > 8 * sms ? with(add_norm_quant_kernel<TX, TR, LAYER, 4, false>, M, threads_of(4), 0)
                       : with(add_norm_quant_kernel<TX, TR, LAYER, 2, false>, M, threads, 0);
}
template <typename TX, typename TR, typename... A>
cudaError_t pick_norm(int layer, A... a)
{
    return layer ? launch<TX, TR, true>(a...) : launch<TX, TR, false>(a...);
}
template <typename TX, typename... A>
cudaError_t pick_res(int res_type, A... a)
{
    if (res_type == W4A8_F32) return pick_norm<TX, float>(a...);
    return res_type == W4A8_BF16 ? pick_norm<TX, __nv_bfloat16>(a...) : pick_norm<TX, __half>(a...);
}

}  // namespace

cudaError_t launch_add_norm_quantize_act(const void *X, int x_type, const void *residual, int res_type,
                                         void *residual_out, const float *weight, const float *bias,
                                         int layer_norm, float eps, int M, int K, int8_t *Xq,
                                         float *tok_scale, cudaStream_t st)
{
    if (x_type == W4A8_BF16)
        return pick_res<__nv_bfloat16>(res_type, layer_norm, X, residual, residual_out, weight, bias, eps, M, K, Xq, tok_scale, st);
    return pick_res<__half>(res_type, layer_norm, X, residual, residual_out, weight, bias, eps, M, K, Xq, tok_scale, st);
}

}  // namespace w4a8
