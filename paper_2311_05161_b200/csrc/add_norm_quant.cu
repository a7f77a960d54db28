// Residual addition, normalisation and token-wise INT8 quantizer in one pass.
//
// Between two sub-blocks of a decoder layer the branch's output joins the residual stream and the
// normalised stream becomes the next linear's INT8 input.  One launch reads the branch and the
// stream once and writes the stream and the codes: 7 bytes per element with a 16-bit stream, 11
// with a 32-bit one, where addition and w4a8_norm_quantize_act apart move 9 (13).  Bound by memory for prompts,
// by the launch and three dependent steps (load, sum, maximum) for a few tokens.
//
// A CTA owns a token and a thread EV vectors of eight of its elements, kept in registers through
// all phases.  The sums are binary64 from the elements on: their order then does not matter to
// the binary32 values that are rounded from them (but for one case in about 2^28), so any
// other implementation in binary64 gives the same codes.
#include "common.cuh"
#include "quant_math.cuh"

namespace w4a8 {

namespace {

// Eight elements as binary32.
template <typename T> struct Vec8;
template <> struct Vec8<__half> {
    static __device__ __forceinline__ void load(const __half *p, float (&x)[8])
    {
        const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(p));
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
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&x)[8])
    {
        const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(p));
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
    static __device__ __forceinline__ void load(const float *p, float (&x)[8])
    {
        const float4 a = __ldcs(reinterpret_cast<const float4 *>(p));
        const float4 b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    static __device__ __forceinline__ void round_store(float *p, float (&x)[8])
    {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};

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

template <typename TX, typename TR, bool LAYER, int EV>
__global__ void __launch_bounds__(512)
add_norm_quant_kernel(const TX *__restrict__ X, const TR *residual, TR *residual_out,
                      const float *__restrict__ weight, const float *__restrict__ bias, float eps,
                      double inv_k, int K, int8_t *__restrict__ Xq, float *__restrict__ tok_scale)
{
    __shared__ double red_mean[16], red_sq[16];
    __shared__ float red_max[16];
    allow_dependents();
    dependent_wait();
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 31, warp = tid >> 5, nwarps = T >> 5;
    const int nvec = K >> 3;
    const size_t row = (size_t)blockIdx.x * K;
    float x[EV][8], y[EV][8];
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int v = tid + i * T;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.0f;
        if (v < nvec) {
            Vec8<TX>::load(X + row + v * 8, y[i]);
            Vec8<TR>::load(residual + row + v * 8, x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int v = tid + i * T;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = __fadd_rn(x[i][e], y[i][e]);
        if (v < nvec) Vec8<TR>::round_store(residual_out + row + v * 8, x[i]);
    }
    if (LAYER) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < EV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += (double)x[i][e];
        const float mu = __double2float_rn(cta_sum(s, red_mean, lane, warp, nwarps) * inv_k);
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
        for (int e = 0; e < 8; ++e) sq = fma((double)x[i][e], (double)x[i][e], sq);
    sq = cta_sum(sq, red_sq, lane, warp, nwarps);
    const float r = __double2float_rn(rsqrt(sq * inv_k + (double)eps));
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int v = tid + i * T;
        if (v < nvec) {
            const float4 wa = __ldg(reinterpret_cast<const float4 *>(weight) + 2 * v);
            const float4 wb = __ldg(reinterpret_cast<const float4 *>(weight) + 2 * v + 1);
            const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = __fmul_rn(__fmul_rn(x[i][e], r), w[e]);
            if (bias) {
                const float4 ba = __ldg(reinterpret_cast<const float4 *>(bias) + 2 * v);
                const float4 bb = __ldg(reinterpret_cast<const float4 *>(bias) + 2 * v + 1);
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
        if (lane == 0) red_max[warp] = amax;
        __syncthreads();
        amax = red_max[0];
        for (int w = 1; w < nwarps; ++w) amax = fmaxf(amax, red_max[w]);
    }
    const float q = amax > 0.0f ? __fdiv_rn(127.0f, amax) : 0.0f;
    if (tid == 0) tok_scale[blockIdx.x] = __fdiv_rn(amax, 127.0f);
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int v = tid + i * T;
        if (v < nvec) *reinterpret_cast<uint2 *>(Xq + row + v * 8) = quantize8(x[i], q);
    }
}

template <typename TX, typename TR, bool LAYER>
cudaError_t launch(const void *X, const void *residual, void *residual_out, const float *weight,
                   const float *bias, float eps, int M, int K, int8_t *Xq, float *tok_scale,
                   cudaStream_t st)
{
    constexpr int EV = 4;
    const int threads = ((K / 8 + EV - 1) / EV + 31) / 32 * 32;
    return launch_overlapped(add_norm_quant_kernel<TX, TR, LAYER, EV>, dim3(M), dim3(threads), 0, st,
                             static_cast<const TX *>(X), static_cast<const TR *>(residual),
                             static_cast<TR *>(residual_out), weight, bias, eps, 1.0 / K, K, Xq, tok_scale);
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
