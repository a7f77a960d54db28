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
//    (expand in kv_attention.cu) where a table lookup would need a table per token.
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

// Sequence of a row: the number of entries among cu_rows[1 .. batch] that are <= row (batch for a
// row behind the last sequence).  All lanes of a warp call it with the same row; every step probes
// 32 places at once, so a batch of 1024 takes two dependent loads.
__device__ __forceinline__ int kv_sequence_of(const KvBatch &bt, int row)
{
    if (!bt.cu_rows) return row;
    const int lane = threadIdx.x & 31;
    int lo = 0, n = bt.batch;                // answer in [lo, lo + n]
    while (n > 0) {
        const int step = (n + 31) >> 5;
        const int at = lo + (lane + 1) * step;              // is cu_rows[at] <= row ?
        const bool le = at <= lo + n && __ldg(bt.cu_rows + at) <= row;
        const int k = __popc(__ballot_sync(0xffffffffu, le));
        lo += k * step;
        n = min(step - 1, n - k * step);
    }
    return lo;
}

// Position of row `row` of sequence b; `ok` false when the length or the offsets make no sense.
__device__ __forceinline__ int kv_position_of(const KvBatch &bt, int b, int row, bool &ok)
{
    const int len = __ldg(bt.kv_lens + b);
    const int begin = bt.cu_rows ? __ldg(bt.cu_rows + b) : b;
    const int end = bt.cu_rows ? __ldg(bt.cu_rows + b + 1) : b + 1;
    ok = len >= 0 && begin >= 0 && begin <= row && end > row && end <= bt.rows;
    return ok ? len - (end - row) : -1;
}

// Page number of position pos (>= 0), or -1.
__device__ __forceinline__ int kv_page_of(const KvCache &c, const KvBatch &bt, int b, int pos)
{
    const int i = pos >> c.page_shift;
    if (i >= bt.max_pages) return -1;
    const int p = __ldg(bt.page_table + (size_t)b * bt.max_pages + i);
    return (unsigned)p < (unsigned)c.num_pages ? p : -1;
}

// Address of the block that holds token slot `slot` of head h of a page.
__device__ __forceinline__ uint8_t *kv_block_at(const KvCache &c, int page, int h, int slot)
{
    return c.pages + (size_t)page * c.page_bytes() +
           ((size_t)h << c.page_shift) * (c.D + 8) + (size_t)(slot >> 4) * kv_block_bytes(c.D);
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
    uint32_t bits = 0x3f800000u;             // 1.0f
    if (raw >= 0x1p-100f) bits = (__float_as_uint(raw) + 8u) & ~15u;
    r = __fdiv_rn(1.0f, __uint_as_float(bits));
    z = (int)fminf(rintf(__fmul_rn(-lo, r)), 13.0f);
    return bits | (uint32_t)z;
}

// Rank of x: Eq. 5 with the levels in ascending order.
__device__ __forceinline__ uint32_t kv_rank(float x, float r, int z)
{
    const float u = __fmul_rn(x, r), a = fabsf(u);
    int l = (int)rintf(u);
    l = min(max(l, -z), 13 - z);
    l += (l > 0) - (l < 0);
    if (a > 0.25f && a <= 0.75f) l = u > 0.0f ? 1 : -1;
    return (uint32_t)(l + z + 1);
}

// Level of a rank in units of the step.
__device__ __forceinline__ float kv_level(uint32_t rank, int z)
{
    const float y = (float)((int)rank - z - 1);
    return y - fminf(fmaxf(0.5f * y, -1.0f), 1.0f);
}

// The eight ranks of a code word in element order, and back.
__device__ __forceinline__ uint32_t kv_half(uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3)
{
    const uint32_t h = r0 | (r1 << 4) | (r2 << 8) | (r3 << 12);
    return ((h << 2) | (h >> 14)) & 0xffffu;
}
__device__ __forceinline__ uint32_t kv_rank_at(uint32_t w, int e)
{
    const uint32_t h = e < 4 ? (w & 0xffffu) : (w >> 16);
    const uint32_t n = (h >> 2) | (h << 14);
    return (n >> (4 * (e & 3))) & 15u;
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
