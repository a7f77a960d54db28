// Rotary positions on queries and keys, and the rows' keys and values into the 4-bit cache, in one pass.
//
// A pair (a, b) of a vector's elements is turned by the angle position * inv_freq:
//   a' = a cos - b sin,  b' = b cos + a sin   (binary32, one rounding per operation),
// Q is rounded once to its 16-bit type, K goes into the quantizer of the cache as it is.  The angle is a product in binary64
// (exact up to positions of 2^29), its fraction of a turn is taken there with 1 / (2 pi) in two parts, and sine and
// cosine come from binary64 and are rounded once: a far position loses nothing, where a binary32 product is off by
// a sixteenth of a radian at 10^6.
//
// As in append, a group of D/8 lanes owns a row and walks over its vectors (queries, keys, values), eight elements a lane.  A
// lane computes four of a row's sines and cosines and gets the other four that it needs from the lane with the other halves of its pairs
// (halves: elements i and i + rotary / 2), whose elements it gets by shuffles too; they stay in registers for all heads.
#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                   // vectors of a group whose loads are in flight together

// Sine and cosine of position * freq, each rounded once from binary64.
__device__ __forceinline__ void turn(int position, float freq, float &s, float &c)
{
    constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
    const double angle = (double)position * (double)freq;
    const double whole = rint(angle * kHi);
    const double part = fma(angle, kLo, fma(angle, kHi, -whole));                // of a turn
    double ds, dc;
    sincospi(2.0 * part, &ds, &dc);
    s = (float)ds;
    c = (float)dc;
}

template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
rope_append_kernel(const RopeArgs a, const KvCache c, int vecs, StatusBlock *sb)
{
    constexpr int LPV = D / 8, GROUPS = kThreads / LPV;
    allow_dependents();
    dependent_wait();
    const int group = threadIdx.x / LPV, l = threadIdx.x % LPV;
    const int row = blockIdx.x * GROUPS + group;
    const int v0 = blockIdx.y * vecs, v1 = min(v0 + vecs, a.q_heads + 2 * c.heads);
    long long slot = row < a.rows ? __ldca(reinterpret_cast<const long long *>(a.slots) + row) : -1;
    if (slot >= (long long)c.num_pages << c.page_shift) {
        if (l == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
        slot = -1;
    }
    const bool here = slot >= 0;
    // ---- this lane's sines and cosines ----
    const int half = a.rotary / 2, lanes = half / 8;           // halves: lanes that hold a first half
    float sn[8], cs[8];
    const bool turned = 8 * l < a.rotary;
    const int partner = INTERLEAVED ? l : l < lanes ? l + lanes : l - lanes;
    if (v0 < a.q_heads + c.heads) {
        // halves: the lane of the first half takes the first four of eight pairs, its partner the others
        const int pair0 = INTERLEAVED ? 4 * l : l < lanes ? 8 * l : 8 * (l - lanes) + 4;
        float s4[4] = {0.0f, 0.0f, 0.0f, 0.0f}, c4[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        if (here && turned) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                int axis = a.pair_axis ? __ldca(a.pair_axis + pair0 + k) : 0;
                if ((unsigned)axis >= (unsigned)a.axes) {
                    report_failure(sb, W4A8_ERR_BAD_TABLE, row);
                    axis = 0;
                }
                turn(__ldca(a.positions + (size_t)axis * a.rows + row), __ldca(a.inv_freq + pair0 + k), s4[k], c4[k]);
            }
        }
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sn[2 * k] = -s4[k];
                sn[2 * k + 1] = s4[k];
                cs[2 * k] = cs[2 * k + 1] = c4[k];
            }
        } else {
            const bool first = l < lanes;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float so = __shfl_sync(0xffffffffu, s4[k], partner, LPV), co = __shfl_sync(0xffffffffu, c4[k], partner, LPV);
                sn[k] = first ? -s4[k] : so;
                sn[4 + k] = first ? -so : s4[k];
                cs[k] = first ? c4[k] : co;
                cs[4 + k] = first ? co : c4[k];
            }
        }
    }
    const T *q_from = static_cast<const T *>(a.Q) + (size_t)row * a.q_stride + 8 * l;
    const T *k_from = static_cast<const T *>(a.K) + (size_t)row * a.k_stride + 8 * l;
    const T *v_from = static_cast<const T *>(a.V) + (size_t)row * a.v_stride + 8 * l;
    T *q_to = static_cast<T *>(a.Q_out) + (size_t)row * a.q_out_stride + 8 * l;
    const int place = (int)(slot & ((1ll << c.page_shift) - 1)), s = place & 15;
    const size_t head_bytes = ((size_t)1 << c.page_shift) * (D + 8);
    uint8_t *block = c.pages + (here ? (size_t)(slot >> c.page_shift) * c.page_bytes() + (size_t)(place >> 4) * kv_block_bytes(D) : 0);
    // (lanes without a row take part in the shuffles)
    auto load = [&](const T *p) { return here ? __ldcs(reinterpret_cast<const uint4 *>(p)) : make_uint4(0u, 0u, 0u, 0u); };
    auto rotate = [&](const uint4 &raw, float (&x)[8]) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t own = (&raw.x)[k];
            const float2 f = to_float2<T>(own);
            x[2 * k] = f.x;
            x[2 * k + 1] = f.y;
            if constexpr (INTERLEAVED) {
                y[2 * k] = f.y;
                y[2 * k + 1] = f.x;
            } else {
                const float2 g = to_float2<T>(__shfl_sync(0xffffffffu, own, partner, LPV));
                y[2 * k] = g.x;
                y[2 * k + 1] = g.y;
            }
        }
        if (turned) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = __fadd_rn(__fmul_rn(x[k], cs[k]), __fmul_rn(y[k], sn[k]));
        }
    };
    // ---- queries ----
    for (int h = v0; h < min(v1, a.q_heads); h += kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j)
            if (h + j < min(v1, a.q_heads)) raw[j] = load(q_from + (size_t)(h + j) * D);
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            if (h + j >= min(v1, a.q_heads)) break;
            float x[8];
            rotate(raw[j], x);
            const uint4 out = {pack2_sat<T>(x[0], x[1]), pack2_sat<T>(x[2], x[3]), pack2_sat<T>(x[4], x[5]), pack2_sat<T>(x[6], x[7])};
            if (here) __stcs(reinterpret_cast<uint4 *>(q_to + (size_t)(h + j) * D), out);
        }
    }
    // ---- keys and values ----
#pragma unroll
    for (int value = 0; value < 2; ++value) {
        const int base = a.q_heads + value * c.heads;
        const int h0 = max(v0 - base, 0), h1 = min(v1 - base, c.heads);
        const T *from = value ? v_from : k_from;
        const int code_at = kv_code_offset(D, value, s, l), word_at = kv_word_offset(D, value, s);
        for (int h = h0; h < h1; h += kUnroll) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j)
                if (h + j < h1) raw[j] = load(from + (size_t)(h + j) * D);
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                if (h + j >= h1) break;
                float x[8];
                if (value == 0) rotate(raw[j], x);
                else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 f = to_float2<T>((&raw[j].x)[k]);
                        x[2 * k] = f.x;
                        x[2 * k + 1] = f.y;
                    }
                }
                float lo = 0.0f, hi = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    lo = min3(lo, x[k], x[k + 1]);
                    hi = max3(hi, x[k], x[k + 1]);
                }
#pragma unroll
                for (int o = LPV / 2; o > 0; o >>= 1) {
                    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
                }
                float r;
                int z;
                const uint32_t word = kv_range_word(lo, hi, r, z), codes = kv_code_word(x, r, z);
                if (here) {
                    uint8_t *to = block + (h + j) * head_bytes;
                    *reinterpret_cast<uint32_t *>(to + code_at) = codes;
                    if (l == 0) *reinterpret_cast<uint32_t *>(to + word_at) = word;
                }
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch(const RopeArgs &a, int interleaved, const KvCache &c, StatusBlock *sb, cudaStream_t st)
{
    // vectors per CTA: all of a row's where the rows alone give eight CTAs per SM, fewer (down to one) else
    const int groups = kThreads / (D / 8), across = (a.rows + groups - 1) / groups, all = a.q_heads + 2 * c.heads;
    const int parts = (8 * device_sms() + across - 1) / across;
    const int vecs = parts >= all ? 1 : (all + parts - 1) / parts;
    const dim3 grid(across, (all + vecs - 1) / vecs);
    return interleaved ? launch_overlapped(rope_append_kernel<T, D, true>, grid, dim3(kThreads), 0, st, a, c, vecs, sb)
                       : launch_overlapped(rope_append_kernel<T, D, false>, grid, dim3(kThreads), 0, st, a, c, vecs, sb);
}

}  // namespace

cudaError_t launch_rope_kv_append(const RopeArgs &a, int bf16, int interleaved, const KvCache &c, StatusBlock *sb,
                                  cudaStream_t st)
{
    if (c.D == 64) return bf16 ? launch<__nv_bfloat16, 64>(a, interleaved, c, sb, st) : launch<__half, 64>(a, interleaved, c, sb, st);
    return bf16 ? launch<__nv_bfloat16, 128>(a, interleaved, c, sb, st) : launch<__half, 128>(a, interleaved, c, sb, st);
}

}  // namespace w4a8
