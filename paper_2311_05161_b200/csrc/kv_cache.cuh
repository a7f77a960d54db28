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

// Page number of position pos (>= 0), or -1.
__device__ __forceinline__ int kv_page_of(const KvCache &c, const KvBatch &bt, int b, int pos)
{
    const int i = pos >> c.page_shift;
    if (i >= bt.max_pages) return -1;
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
// -z before rounding.  y is the smaller of rint(f |u|) and rint|u| + 1, where f is the binary32 number in front of 2 (with 2
// itself, 3/4 would be a tie): equal to the definition for every binary32 |u| below 16.  Rounding and conversion are additions of 1.5 * 2^23 (minus one), which leave the integer in the mantissa's low bits (the
// constant's own low 16 bits are zero).
__device__ __forceinline__ uint32_t kv_rank_bits(float x, float r, float top, float bias)
{
    const float u = __fmul_rn(x, r);
    const float y = __fadd_rn(fminf(__fmaf_rn(fabsf(u), 0x1.fffffep0f, 12582911.0f), __fadd_rn(fabsf(u), 12582912.0f)), -12582911.0f);
    return __float_as_uint(__fadd_rn(fminf(copysignf(y, u), top), bias));
}
__device__ __forceinline__ uint32_t kv_code_word(const float (&x)[8], float r, int z)
{
    const float top = (float)(14 - z), bias = 12582913.0f + (float)z;
    uint32_t k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = kv_rank_bits(x[i], r, top, bias);
    const uint32_t lo = (k[3] * 16u + k[2]) * 256u + (k[1] * 16u + k[0]);
    const uint32_t hi = (k[7] * 16u + k[6]) * 256u + (k[5] * 16u + k[4]);
    const uint32_t w = __byte_perm(lo, hi, 0x5410);
    return ((w << 2) & 0xFFFCFFFCu) | ((w >> 14) & 0x00030003u);         // both halves rotated left by two
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

cudaError_t launch_kv_append(const void *K, const void *V, int bf16, long long k_stride,
                             long long v_stride, const KvCache &c, const KvBatch &bt,
                             StatusBlock *sb, cudaStream_t st);
cudaError_t launch_kv_read(const KvCache &c, const KvBatch &bt, void *K, void *V, int bf16,
                           StatusBlock *sb, cudaStream_t st);

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
};
size_t kv_attention_workspace(int rows, int batch, int q_heads, int kv_heads, int D);
cudaError_t launch_kv_attention(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st);

}  // namespace w4a8
