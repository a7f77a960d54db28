// Shared by the two attention kernels over the 4-bit cache (kv_attention.cu: few rows per sequence;
// kv_prefill.cu: many): waits, the expansion of the codes, sequences as the kernels see them.
#pragma once

#include "kv_cache.cuh"

namespace w4a8 {

constexpr unsigned long long kWaitNs = 2000000000ull;      // limit of every bounded wait
constexpr uint32_t kSuspendHintNs = 20000;                 // a waiting thread is woken when the phase completes; until then it stays out of the issue slots
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoReference = -3.402823466e38f;           // below every score: of a row that has seen no key
constexpr float kSlack = 15.0f;                            // weights stay below 2^15, within binary16
// A reference that moves is put this far below the largest exponent, so that weights down to 2^-29 of the largest
// one are more than binary16's zero: a hundred thousand of those add up to 2^-12 of it, half a step of a weight.
// (Every bit of it is one less above, for what comes later; 7 bits cost the many-row form 4 % in moved references.)
constexpr float kRoom = 4.0f;
// The denominator sums weight / step, up to 2^(15 + 100) each.  A reference also moves, by kShift, where a sum has passed
// kFull: a hundred more stay below 2^122.  Where sums are joined, large ones are taken against a
// reference kLift higher first.
constexpr float kFull = 0x1p100f, kShift = 16.0f, kLift = 20.0f;

__device__ __forceinline__ uint32_t smem_addr(const void *p)
{
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(kSuspendHintNs)
        : "memory");
    return ok != 0;
}
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity)
{
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
    do {
        if (try_wait(bar, parity)) return true;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    } while (t - t0 < kWaitNs);
    return false;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t perm(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
    return d;
}
__device__ __forceinline__ uint32_t hfma2_sat(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.sat.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t pack_half2(float a, float b)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
constexpr uint32_t kNibble = 0x03C003C0u;    // bits 6-9 of both halves
constexpr uint32_t kMinusEight = 0xC800C800u, kSixteen = 0x4C004C00u;
constexpr uint32_t kMinusHalf = 0xB800B800u, kQuarter = 0x34003400u, kMinusQuarter = 0xB400B400u;

// The constant of the saturated term, 1/4 - (16 + z) / 4, from a pair of binary16 numbers 16 + z.
__device__ __forceinline__ uint32_t sat_constant(uint32_t off) { return hfma2(off, kMinusQuarter, kQuarter); }

// The four ranks of each 16-bit half of w -> four pairs (rank k of the low half, of the high half):
// -(level + 16 + z) / 2.
// Mask and magic number come in registers that the compiler cannot see through: one logic
// instruction per pair, where two immediates would take two.
struct ExpandConsts {
    uint32_t nibble, minus_eight;
};
__device__ __forceinline__ uint32_t pick_rank(uint32_t x, const ExpandConsts &k)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(x), "r"(k.nibble), "r"(k.minus_eight));   // (x & b) | c
    return d;
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ void expand(uint32_t w, uint32_t c, const ExpandConsts &k, uint32_t (&o)[4])
{
    uint32_t lin[4];
    const uint32_t sw = perm(w, w, 0x2301u);         // the bytes of each half swapped
    lin[0] = pick_rank(w << 4, k);
    lin[1] = pick_rank(w, k);
    lin[2] = pick_rank(sw << 4, k);
    lin[3] = pick_rank(sw, k);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = hadd2(lin[i], hfma2_sat(lin[i], kMinusHalf, c));
}

// Quotient by a number that the launch fixes: n / d for n < 2^31 (d < 2^16) by one multiplication with
// ceil(2^(31 + s) / d), 2^s >= d.
struct Divisor {
    uint32_t d, mul, shift;
    explicit Divisor(uint32_t v) : d(v), shift(0)
    {
        while ((1u << shift) < v) ++shift;
        mul = (uint32_t)(((1ull << (31 + shift)) + v - 1) / v);
    }
    __device__ __forceinline__ int div(int n) const
    {
        return (int)(((unsigned long long)(uint32_t)n * mul) >> (31 + shift));
    }
};

// 64-bit quotient that takes the 32-bit path when it can.
__device__ __forceinline__ long long quotient(long long a, long long b)
{
    if (((unsigned long long)(a | b) >> 32) == 0) return (long long)((uint32_t)a / (uint32_t)b);
    return a / b;
}

// One sequence of the batch, its numbers checked.
struct Seq {
    int row0, n, len;          // rows of the call, tokens
};
__device__ __forceinline__ Seq load_seq(const KvAttnArgs &a, int b, StatusBlock *sb)
{
    const KvBatch &bt = a.batch;
    Seq s;
    s.len = __ldca(bt.kv_lens + b);
    s.row0 = bt.cu_rows ? __ldca(bt.cu_rows + b) : b;
    const int row1 = bt.cu_rows ? __ldca(bt.cu_rows + b + 1) : b + 1;
    s.n = row1 - s.row0;
    const int most = bt.max_pages << a.cache.page_shift;
    if (s.len < 0 || s.len > most || s.row0 < 0 || row1 > bt.rows || row1 < s.row0) {
        report_failure(sb, W4A8_ERR_BAD_TABLE, b);
        s.len = min(max(s.len, 0), most);
        if (s.row0 < 0 || row1 > bt.rows || row1 < s.row0) s.n = 0;
    }
    return s;
}

// Rows i_first .. i_last of a sequence (rows of one tile): a row sees keys [lo, hi); one in front of
// position 0 sees none.
struct Sight {
    int pos0, len, window;
    bool causal;
    __device__ Sight(const KvAttnArgs &a, const Seq &s) : pos0(s.len - s.n), len(s.len), window(a.window), causal(a.causal != 0) {}
    __device__ int hi(int i) const { return pos0 + i < 0 ? 0 : causal ? pos0 + i + 1 : len; }
    __device__ int lo(int i) const { return window > 0 ? (int)max(0ll, (long long)pos0 + i + 1 - window) : 0; }
};

// Counters of shared items in the workspace, behind the status block.  Both kernels use this region and
// leave it zero, so that calls of either kind can follow each other on one workspace.
constexpr int kCountersPerSm = 8;
inline size_t kv_counters_bytes(int sms) { return align_up((size_t)sms * kCountersPerSm * sizeof(int), 256); }

// What the prefill kernel's launcher needs (kv_prefill.cu).
size_t kv_prefill_workspace(int D);
cudaError_t launch_kv_prefill(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st);

}  // namespace w4a8
