// The paged dINT4 key / value cache: layout, batch description, one vector's quantizer and
// expansion.  The layout is stated in include/w4a8.h; the reasons for it are here.
//
//  - A block of 16 tokens of one head (16 (D + 8) bytes: 2176 for D = 128) is contiguous, so the
//    attention kernel brings both operands and their words with one bulk copy, and a page's
//    blocks of a head are adjacent.
//  - Key codes lie token by token: the score product contracts over D, whose order inside an MMA
//    operand is free, so a thread takes 16 consecutive bytes of a token as its operand words.
//  - Value codes lie as [half][slice][token][bytes]: the value product contracts over tokens, an
//    MMA operand register holds the same element of two neighbouring tokens, and this order lets a
//    thread load its slice of a token pair with one 16-byte access, without bank conflicts.
//  - A code is a rank i = y + z + 1, where y is the level x for |x| < 1 doubled and moved out by one
//    for |x| >= 1: the level is y - clamp(y / 2, -1, 1), three packed binary16 operations
//    (expand in kv_attention.cuh) where a table lookup would need a table per token.
//  - The ranks of a 16-bit half are rotated left by two bits: two of them then lie at bits 2-5 and
//    6-9, inside the mantissa of a binary16 number, and swapping the half's bytes brings the
//    other two there.
#pragma once

#include "common.cuh"

namespace w4a8 {

constexpr int kKvBlock = 16;                 // tokens per block

__host__ __device__ inline int kv_block_bytes(int D) { return kKvBlock * (D + 8); }

struct KvBatch {
    const int32_t *page_table;               // [batch][max_pages]
    const int32_t *kv_lens;                  // [batch]
    const int32_t *cu_rows;                  // [batch + 1] or NULL
    int max_pages, batch, rows;
};

struct KvCache {
    uint8_t *pages;
    int num_pages, page_shift;               // page_size = 1 << page_shift
    int heads, D;
    __host__ __device__ size_t page_bytes() const
    {
        return ((size_t)heads << page_shift) * (D + 8);
    }
};

// Position of row `row` of sequence b; `ok` false when the length or the offsets make no sense.
__device__ __forceinline__ int kv_position_of(const KvBatch &bt, int b, int row, bool &ok)
{
    const int len = __ldca(bt.kv_lens + b);
    const int begin = bt.cu_rows ? __ldca(bt.cu_rows + b) : b;
    const int end = bt.cu_rows ? __ldca(bt.cu_rows + b + 1) : b + 1;
    ok = len >= 0 && begin >= 0 && begin <= row && end > row && end <= bt.rows;
    return ok ? len - (end - row) : -1;
}

// Page number of position pos, or -1 (as of a position in front of the sequence or behind its table).
__device__ __forceinline__ int kv_page_of(const KvCache &c, const KvBatch &bt, int b, int pos)
{
    const int i = pos >> c.page_shift;
    if ((unsigned)i >= (unsigned)bt.max_pages) return -1;
    const int p = __ldca(bt.page_table + (size_t)b * bt.max_pages + i);
    return (unsigned)p < (unsigned)c.num_pages ? p : -1;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float d;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Byte offset, inside a block, of the word with the codes of elements 8 w .. 8 w + 7 of token s.
__device__ __forceinline__ int kv_code_offset(int D, int is_value, int s, int w)
{
    if (!is_value) return s * (D / 2) + 4 * w;
    const int cb = D / 16;                   // bytes of a slice: 4 or 8
    const int slice = (4 * w) / cb;
    return 8 * D + (((s >> 3) * 8 + slice) * 8 + (s & 7)) * cb + (4 * w) % cb;
}
__device__ __forceinline__ int kv_word_offset(int D, int is_value, int s)
{
    return 16 * D + 64 * is_value + 4 * s;
}

// Step and zero-point of a vector with range [lo, hi] (lo <= 0 <= hi), as the stored word.
__device__ __forceinline__ uint32_t kv_range_word(float lo, float hi, float &r, int &z)
{
    const float raw = __fdiv_rn(__fsub_rn(__fmul_rn(hi, 0.5f), __fmul_rn(lo, 0.5f)), 6.5f);
    // A vector of zeros gets a step far below any that matters: attention takes a value's step for the size of what the
    // token adds to the output (with a step of 1, a token of high score and zero value pushed the weights of values of
    // 2^-14 below binary16).  Not smaller still, so that the token's part of the denominator, a weight times 1 / step,
    // keeps 60 bits below the weights of values as large as binary16 holds.
    uint32_t bits = 0x1f800000u;             // 2^-64
    if (raw >= 0x1p-100f) bits = (__float_as_uint(raw) + 8u) & ~15u;
    r = __fdiv_rn(1.0f, __uint_as_float(bits));
    z = (int)fminf(rintf(__fmul_rn(-lo, r)), 13.0f);
    return bits | (uint32_t)z;
}

// Eight consecutive elements as a code word: Eq. 5, the levels numbered in ascending order.  With u = x r, the place y
// of a level counted from zero is 0 for |u| <= 1/4, +-1 for |u| <= 3/4 (the specials) and
// +-(rint|u| + 1) beyond; the rank is y + z + 1.  The clamp of Eq. 5 acts at the upper end only: the least element's u is
// -z before rounding.  y is the one of rint(f u), rint(u) - 1 and rint(u) + 1 that lies between the others, where f is the binary32
// number in front of 2 (with 2 itself, 3/4 would be a tie): equal to the definition for every binary32 |u| below 16.  Rounding and
// conversion are additions of 1.5 * 2^23, which leave the integer in the mantissa's low bits (the constant's own low 16 bits
// are zero); from there on two elements share an instruction.  (In binary32 throughout: eight instructions per element, here five.)
__device__ __forceinline__ uint32_t kv_two_ranks(float x0, float x1, float r, uint32_t zz)
{
    const float u0 = __fmul_rn(x0, r), u1 = __fmul_rn(x1, r);
    const uint32_t twice = __byte_perm(__float_as_uint(__fmaf_rn(u0, 0x1.fffffep0f, 12582912.0f)), __float_as_uint(__fmaf_rn(u1, 0x1.fffffep0f, 12582912.0f)), 0x5410);
    const uint32_t once = __byte_perm(__float_as_uint(__fadd_rn(u0, 12582912.0f)), __float_as_uint(__fadd_rn(u1, 12582912.0f)), 0x5410);
    const uint32_t y = __viaddmin_s16x2(once, 0x00010001u, __viaddmax_s16x2(once, 0xffffffffu, twice));
    return __viaddmin_s16x2(y, zz, 0x000f000fu);
}
// zz = z + 1 in both halves.
__device__ __forceinline__ uint32_t kv_code_word(const float (&x)[8], float r, uint32_t zz)
{
    const uint32_t lo = kv_two_ranks(x[1], x[3], r, zz) * 16u + kv_two_ranks(x[0], x[2], r, zz);
    const uint32_t hi = kv_two_ranks(x[5], x[7], r, zz) * 16u + kv_two_ranks(x[4], x[6], r, zz);
    const uint32_t w = __byte_perm(lo, hi, 0x6420);
    return ((w << 2) & 0xFFFCFFFCu) | ((w >> 14) & 0x00030003u);         // both halves rotated left by two
}
__device__ __forceinline__ uint32_t kv_twice(int z) { return (uint32_t)(z + 1) * 0x00010001u; }

// The words of four vectors whose elements LPV lanes hold, from the lanes' ranges: the four are reduced side by side, so that a lane
// is left with one vector's and the divisions of a step are done once for four.  Vector j's lanes: kv_owner_of(j) and the LPV / 4 - 1 behind it.
template <int LPV> __device__ __forceinline__ int kv_owner_of(int j) { return (j >> 1) * (LPV / 2) + (j & 1) * (LPV / 4); }
template <int LPV>
__device__ __forceinline__ uint32_t kv_four_words(float (&lo)[4], float (&hi)[4], int lane, float &r, int &z)
{
    constexpr int A = LPV / 2, B = LPV / 4;
    const bool up_a = lane & A, up_b = lane & B;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float send_lo = up_a ? lo[j] : lo[j + 2], send_hi = up_a ? hi[j] : hi[j + 2];
        lo[j] = fminf(up_a ? lo[j + 2] : lo[j], __shfl_xor_sync(0xffffffffu, send_lo, A));
        hi[j] = fmaxf(up_a ? hi[j + 2] : hi[j], __shfl_xor_sync(0xffffffffu, send_hi, A));
    }
    const float send_lo = up_b ? lo[0] : lo[1], send_hi = up_b ? hi[0] : hi[1];
    float l = fminf(up_b ? lo[1] : lo[0], __shfl_xor_sync(0xffffffffu, send_lo, B));
    float h = fmaxf(up_b ? hi[1] : hi[0], __shfl_xor_sync(0xffffffffu, send_hi, B));
#pragma unroll
    for (int o = B / 2; o > 0; o >>= 1) {
        l = fminf(l, __shfl_xor_sync(0xffffffffu, l, o));
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, o));
    }
    return kv_range_word(l, h, r, z);
}

// The eight levels of a code word, halved: pair k holds elements k and k + 4.  (x = rank - z - 1;
// level / 2 = (x + 1) / 2 - sat(x / 4 + 1/2), packed binary16, exact.)
__device__ __forceinline__ void kv_levels(uint32_t w, int z, __half2 (&o)[4])
{
    const uint32_t off = (uint32_t)z * 0x00400040u + 0x48004800u;        // (16 + z) / 2 twice
    const uint32_t sw = __byte_perm(w, w, 0x2301);
    const uint32_t bits[4] = {w << 4, w, sw << 4, sw};
    const __half2 minus_half = __float2half2_rn(-0.5f), quarter = __float2half2_rn(0.25f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lin = (bits[k] & 0x03C003C0u) | 0xC800C800u;      // -(16 + rank) / 2
        const __half2 x = __hadd2(*reinterpret_cast<const __half2 *>(&lin), *reinterpret_cast<const __half2 *>(&off));
        o[k] = __hsub2(__hneg2(x), __hfma2_sat(x, minus_half, quarter));
    }
}

template <typename T> __device__ __forceinline__ float2 to_float2(uint32_t v);
template <> __device__ __forceinline__ float2 to_float2<__half>(uint32_t v)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}
template <> __device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

cudaError_t launch_kv_append(const void *K, const void *V, int bf16, long long k_stride,
                             long long v_stride, const KvCache &c, const KvBatch &bt,
                             StatusBlock *sb, cudaStream_t st);
cudaError_t launch_kv_read(const KvCache &c, const KvBatch &bt, void *K, void *V, int bf16,
                           StatusBlock *sb, cudaStream_t st);

// Rotary positions: element pairs of the first `rotary` elements, turned by position[axis of the pair] * inv_freq[pair].
struct RopeArgs {
    const void *Q, *K, *V;
    long long q_stride, k_stride, v_stride;
    const int32_t *positions;                // [axes][rows]
    const int32_t *pair_axis;                // [rotary / 2] or NULL: axis 0
    const float *inv_freq;                   // [rotary / 2]
    void *Q_out;
    long long q_out_stride;
    const int64_t *slots;                    // [rows]: page * page_size + place, negative: no row
    int axes, rotary, rows, q_heads;
};
cudaError_t launch_rope_kv_append(const RopeArgs &a, int bf16, int interleaved, const KvCache &c, StatusBlock *sb,
                                  cudaStream_t st);

// Accepted drafted rows, as places among the sequence's rows of the call.
struct KvPaths {
    const int32_t *accepted;                 // [batch][most]
    const int32_t *accept_lens;              // [batch]
    const int32_t *kept;                     // [batch] or NULL: lengths of sequences without rows in the call
    int32_t *kv_lens_out;                    // [batch] or NULL
    int most;
};
cudaError_t launch_kv_accept(const KvCache &c, const KvBatch &bt, const KvPaths &paths, StatusBlock *sb, cudaStream_t st);

// A step's plan.
struct KvPlanArgs {
    const int32_t *held, *kv_lens, *add;     // [batch]
    int32_t *page_table;                     // [batch][max_pages]
    int32_t *free_pages;                     // [num_pages]
    const int32_t *free_count;
    int32_t *free_count_out, *kv_lens_out, *cu_rows, *positions;
    int64_t *slots;
    int batch, max_pages, page_shift, num_pages, rows;
    bool wide_stores;                        // positions and slots take 16-byte stores
};
constexpr int kPlanMaxBatch = 8192;        // 24 bytes each in shared memory
cudaError_t launch_kv_plan(const KvPlanArgs &a, StatusBlock *sb, int *ticket, cudaStream_t st);

struct KvAttnArgs {
    const void *Q;
    int q_bf16;
    long long q_stride;
    KvCache cache;
    KvBatch batch;
    int q_heads;
    float scale;
    int causal, window;
    void *O;
    int o_bf16;
    float *lse;
    // the extended form only
    int sinks;                               // first tokens that stay visible beside the window
    const uint32_t *tree;                    // [rows][tree_words] or NULL: drafted rows that a row sees
    int tree_words;
};
size_t kv_attention_workspace(int rows, int batch, int q_heads, int kv_heads, int D);
cudaError_t launch_kv_attention(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st);

}  // namespace w4a8
