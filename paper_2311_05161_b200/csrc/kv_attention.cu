// Attention over the 4-bit cache, decode form: a few query rows per sequence, many keys.
//
// The work is one scan of the cached blocks (16 tokens of one head, 2176 bytes for D = 128), each
// expanded once from 4 bits to binary16 in registers and used twice on the tensor cores: the scores
// S^T = K Q^T (tokens x query rows) and the output O^T = V^T P^T (elements x query rows), both with
// mma.m16n8k16, so that up to eight query rows (the heads that share a key head, times the rows
// of a sequence) ride on one expansion.  With the cache as the MMA's 16-row operand no part of the
// instruction is spent on padding the few rows to 16, and a thread owns one or two tokens, whose
// zero-points are then plain register constants.
//
// Expansion of eight codes (one word): with x = i - z - 1 for rank i, the level is
// x - 2 sat(x / 4 + 1/2) + 1.  Seven logic instructions put each rank into the mantissa of
// lin = -(16 + i) / 2 (binary16), one packed fma.sat per pair makes the saturated term, one packed
// addition joins the two: -2 (lin + sat) = level + 16 + z.  The factor goes into the scale, the offset is
// a constant per token: the score accumulator starts from it times sum(q), and one extra MMA per block
// sums (16 + z) p for the output.  What bounds the kernel is this expansion: packed binary16 and logic
// instructions issue at half rate and overlap only in part, some 26 cycles per word and scheduler (30
// with the MMA) where the memory would allow 23; measured in a loop of its own.  (Leaving the
// addition to the tensor cores, as a second operand, takes the same time for one row tile and more for two.)
// Softmax: the weight of token j for the value product is 2^(s_j + log2(step_j) - m), with the value's
// step folded into the exponent, so that it fits binary16 whatever the steps' sizes; the
// denominator sums 2^(s_j - m) in binary32.  m is a running reference and no exact maximum: it moves
// only when a weight would exceed 2^15 (one vote per 32 tokens instead of a reduction).
//
// Schedule: the blocks of all (sequence, key head, row tile) items form one list, which the
// CTAs share evenly whatever the lengths are (every CTA computes the list's prefix sums from the
// lengths on the device); an item that several CTAs share leaves partial results in the
// workspace and the last of them to finish joins all parts in list order, so the result does not
// depend on who is last.  Inside a CTA the warps take blocks in turn, each with its own ring of
// bulk copies.
//
// Measured (8 key heads of 128 unless said): 64 ragged sequences of 1000 to 6000 tokens, 8 query heads per key
// head, 248 MB: 80 us, 3.1 TB/s, issue slots 66 %, binary16 pipe 53 %, logic pipe 48 % busy.  One sequence of
// 131001 tokens 52.8 us; 32 ragged sequences with 32 heads of their own 56.1 us; 513 tokens 9.2 us.  Beside the main
// loop (some 36 us of the 52.8 us, at 1200 cycles per 32 tokens and scheduler) stand 8 us until the first
// unit is there (place on the list, page numbers, queries, copies, each waiting for the one before) and 4 us for the joins.
#include "kv_attention.cuh"

namespace w4a8 {

namespace {

constexpr int kWaitSite = 900;
constexpr int kLead = 8;                                   // an item's fixed cost, in units of 32 tokens

__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_block(uint32_t dst, const uint8_t *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2,
                                      const uint32_t a3, const uint32_t b0, const uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What one launch needs beside the arguments.
struct Schedule {
    StatusBlock *sb;
    int *counters;             // [workers]
    float *partials;           // [workers][2] parts of R * (D + 2) numbers
    int min_units;             // least share of a CTA
    int lead;                  // what an item costs beside its units, in units
    Divisor group;             // query heads per key head
};

// One sequence's part of the work list.
struct Part : Seq {
    int first, units;          // units of 32 tokens that any of its rows can see
    int tiles;                 // row tiles per key head
    // length of the work list: an item is `lead` places and then its units, at least one
    __device__ int item_length(int lead) const { return lead + max(units, 1); }
    __device__ long long list_length(int heads, int lead) const
    {
        return n > 0 ? (long long)heads * tiles * item_length(lead) : 0;
    }
};

template <int R>
__device__ __forceinline__ Part load_part(const KvAttnArgs &a, int b, int group, StatusBlock *sb)
{
    Part s;
    static_cast<Seq &>(s) = load_seq(a, b, sb);
    s.first = Sight(a, s).lo(0) >> 5;
    s.units = max(0, ((s.len + 31) >> 5) - s.first);
    s.tiles = (int)(((long long)s.n * group + R - 1) / R);
    return s;
}

// The lanes that share a row's elements.
__device__ __forceinline__ uint32_t row_lanes(int lane, int per_row)
{
    return ((1u << per_row) - 1u) << (lane / per_row * per_row);
}

template <int D, int NT, int WARPS>
struct Shape {
    static constexpr int R = 8 * NT;                       // query rows of a tile
    static constexpr int kBlockBytes = 16 * (D + 8);
    static constexpr int kUnitBytes = 2 * kBlockBytes;     // 32 tokens
    static constexpr int kStages = D == 128 ? 3 : 5;       // units in flight per warp
    static constexpr int kRing = WARPS * kStages * kUnitBytes;
    static constexpr int kPad = D + 4;
    static constexpr int kJoin = WARPS * R * kPad * 4;     // overlays the ring between items
    static constexpr int kBig = kRing > kJoin ? kRing : kJoin;
    static constexpr int kSmem = (kBig + WARPS * kStages * 8 + 127) / 128 * 128;
    static constexpr int kCtas = NT == 1 ? 16 / WARPS : 12 / WARPS;
    static_assert(kCtas * (kSmem + 5 * 1024) <= 232448, "shared memory of an SM");
};

template <int D, int NT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, Shape<D, NT, WARPS>::kCtas)
kv_decode_kernel(const KvAttnArgs a, const Schedule sc)
{
    using S = Shape<D, NT, WARPS>;
    constexpr int R = S::R, KW = D / 32, KT = D / 16, BB = S::kBlockBytes, UB = S::kUnitBytes, THREADS = WARPS * 32, LPV = D / 8;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long warp_units[WARPS], found_off;
    __shared__ int found_b, last_part;
    __shared__ float row_m[WARPS][R], row_l[WARPS][R], tile_m[R], tile_l[R];
    __shared__ int row_hi[R], row_lo[R];
    __shared__ __align__(16) uint4 q_frag[NT][KW][32];
    __shared__ float q_sum[R], q_unit[R];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_addr(smem) + warp * S::kStages * UB;
    const uint8_t *ring_ptr = smem + warp * S::kStages * UB;
    const uint32_t bars = smem_addr(smem) + S::kBig + warp * S::kStages * 8;
    if (lane < S::kStages) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + lane * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    allow_dependents();
    dependent_wait();

    const KvBatch &bt = a.batch;
    const int heads = a.cache.heads, group = (int)sc.group.d;
    // ---- this CTA's share of the work list ----
    const int chunk = (bt.batch + THREADS - 1) / THREADS;
    const int b_first = min(bt.batch, tid * chunk), b_last = min(bt.batch, b_first + chunk);
    long long mine = 0;
    for (int b = b_first; b < b_last; ++b) mine += load_part<R>(a, b, group, sc.sb).list_length(heads, sc.lead);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) warp_units[warp] = incl;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) incl += warp_units[w];
        total += warp_units[w];
    }
    const long long per = max(quotient(total + gridDim.x - 1, gridDim.x), (long long)sc.min_units);
    const long long begin = (long long)blockIdx.x * per, end = min(total, begin + per);
    if (begin >= total) return;
    if (begin >= incl - mine && begin < incl) {
        long long at = incl - mine;
        for (int b = b_first; b < b_last; ++b) {
            const long long u = load_part<R>(a, b, group, sc.sb).list_length(heads, sc.lead);
            if (begin < at + u) {
                found_b = b;
                found_off = begin - at;
                break;
            }
            at += u;
        }
    }
    __syncthreads();
    int b = found_b;
    long long off = found_off;             // units of sequence b in front of this CTA's next one
    int stage = 0;
    uint32_t parity = 0;
    bool dead = false;                     // a copy did not arrive in time: nothing more is requested

    for (long long u = begin; u < end;) {
        const Part s = load_part<R>(a, b, group, sc.sb);
        const long long all = s.list_length(heads, sc.lead);
        if (off >= all) {
            off -= all;
            ++b;
            continue;
        }
        const int length = s.item_length(sc.lead), item_units = length - sc.lead;
        const int item = (int)quotient(off, length), at = (int)(off - (long long)item * length);
        const int h = (int)quotient(item, s.tiles), tile = item - h * s.tiles;
        // this CTA's units [in_item, in_item + count) of the item
        const int here = (int)min((long long)(length - at), end - u);
        const int in_item = max(at - sc.lead, 0), count = max(at + here - sc.lead, 0) - in_item;
        const long long first_unit = u - at + sc.lead;       // the item's units on the list
        u += here;
        off += here;
        if (count <= 0) continue;          // its share ends inside the item's lead
        const bool whole = count == item_units;

        // rows of this tile: r = tile * R + i is row r / group of the sequence, query head r % group
        const int rows_here = (int)min((long long)R, (long long)s.n * group - (long long)tile * R);
        const int i_first = sc.group.div(tile * R), i_last = sc.group.div(tile * R + rows_here - 1);
        const Sight sight(a, s);
        const int hi_max = sight.hi(i_last), hi_min = sight.hi(i_first);
        const int lo_min = sight.lo(i_first), lo_max = sight.lo(i_last);
        if (tid < R) {
            const int i = sc.group.div(tile * R + tid);
            row_hi[tid] = tid < rows_here ? sight.hi(i) : s.len;
            row_lo[tid] = tid < rows_here ? sight.lo(i) : 0;
        }
        // units of the share that some row of the tile sees, and this warp's among them
        const int k0 = max(s.first + in_item, lo_min >> 5);
        const int k1 = min(s.first + min(in_item + count, s.units), (hi_max + 31) >> 5);
        const int nk = k1 > k0 + warp ? (k1 - k0 - warp + WARPS - 1) / WARPS : 0;
        const int last_block = (s.len - 1) >> 4;
        const int32_t *table = bt.page_table + (size_t)b * bt.max_pages;
        const uint8_t *head_base = a.cache.pages + ((size_t)h << a.cache.page_shift) * (D + 8);
        const int page_bits = a.cache.page_shift - 4, in_page = (1 << page_bits) - 1;   // in blocks
        const size_t page_bytes = a.cache.page_bytes();
        // byte offsets of the blocks of this warp's next 16 units: lane 2 i + j has block j of the i-th (a block behind
        // the sequence's end, or in front of what the tile sees: its neighbour again; its page may be gone)
        size_t where = 0;
        int requested = 0;                 // units of this item whose copies were started
        auto look_up = [&](int k) {
            const int blk = max(min(2 * (k0 + warp + (k + (lane >> 1)) * WARPS) + (lane & 1), last_block), lo_min >> 4);
            int page = __ldca(table + (blk >> page_bits));
            if ((unsigned)page >= (unsigned)a.cache.num_pages) {
                report_failure(sc.sb, W4A8_ERR_BAD_TABLE, b);
                page = 0;
            }
            where = (size_t)page * page_bytes + (size_t)(blk & in_page) * BB;
        };
        auto request = [&](int k, int st) {  // copy this warp's unit k into ring slot st
            if ((k & 15) == 0) look_up(k);
            if (dead) return;
            ++requested;
            const size_t from = __shfl_sync(0xffffffffu, where, 2 * (k & 15) + (lane & 1));
            if (lane == 0) expect_bytes(bars + st * 8, UB);
            __syncwarp();
            if (lane < 2) copy_block(ring + st * UB + lane * BB, head_base + from, BB, bars + st * 8);
        };
        // ---- queries, shared by the warps: a lane takes eight elements of a row, scales them by a power of two
        // to the top of binary16's range and leaves them as the four pairs that expand() gives of a word ----
        // (Loaded in front of the first copies: 3 units of every warp are 31 MB, and the loads would wait behind them.)
        constexpr int kPass = WARPS * (32 / LPV), kPasses = (R + kPass - 1) / kPass;
        uint4 q_raw[kPasses];
#pragma unroll
        for (int n = 0; n < kPasses; ++n) {
            const int r = warp * (32 / LPV) + lane / LPV + n * kPass;
            const int i = sc.group.div(tile * R + r), head = h * group + tile * R + r - i * group;
            q_raw[n] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows_here)
                q_raw[n] = __ldca(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.Q) + (size_t)(s.row0 + i) * a.q_stride +
                                                                 (size_t)head * D) + lane % LPV);
        }
        {
            int st = stage;
            for (int k = 0; k < min(nk, S::kStages); ++k) {
                request(k, st);
                st = st + 1 == S::kStages ? 0 : st + 1;
            }
        }
#pragma unroll
        for (int n = 0; n < kPasses; ++n) {
            const int r = warp * (32 / LPV) + lane / LPV + n * kPass;
            if (r >= R) break;             // (whole row groups of lanes)
            float f[8], amax = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t v = (&q_raw[n].x)[k];
                if (a.q_bf16) {
                    f[2 * k] = __uint_as_float(v << 16);
                    f[2 * k + 1] = __uint_as_float(v & 0xffff0000u);
                } else {
                    const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&v));
                    f[2 * k] = x.x;
                    f[2 * k + 1] = x.y;
                }
                amax = fmaxf(amax, fmaxf(fabsf(f[2 * k]), fabsf(f[2 * k + 1])));
            }
#pragma unroll
            for (int o = LPV / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(row_lanes(lane, LPV), amax, o));
            // amax * 2^-e in [2^14, 2^15); amax >= 2^-126 or 0, both factors normal
            const int e = min(max((int)((__float_as_uint(amax) >> 23) & 255u) - 127 - 14, -100), 113);
            const float down = __uint_as_float((uint32_t)(127 - e) << 23);
            uint4 pairs;
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t v = pack_half2(f[k] * down, f[k + 4] * down);
                (&pairs.x)[k] = v;
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&v));
                sum += x.x + x.y;
            }
#pragma unroll
            for (int o = LPV / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(row_lanes(lane, LPV), sum, o);
            const int l = lane % LPV;      // the MMA lane that takes these elements: row r % 8, quarter l / KW
            q_frag[r / 8][l % KW][(r % 8) * 4 + l / KW] = pairs;
            if (l == 0) {
                q_sum[r] = 0.5f * sum;
                q_unit[r] = -2.0f * (a.scale * kLog2e) * __uint_as_float((uint32_t)(127 + e) << 23);
            }
        }
        __syncthreads();                   // also row_hi, row_lo
        float qsum[NT][2], unit[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                qsum[n][j] = q_sum[n * 8 + 2 * t + j];
                unit[n][j] = q_unit[n * 8 + 2 * t + j];
            }
        float o[NT][KT][4], osum[NT][4], ref[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][i][j] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) osum[n][j] = 0.0f;
            ref[n][0] = ref[n][1] = kNoReference;
            l[n][0] = l[n][1] = 0.0f;
        }
        ExpandConsts ek = {kNibble, kMinusEight};
        asm volatile("" : "+r"(ek.nibble), "+r"(ek.minus_eight));
        const uint32_t only_g0 = g == 0 ? 0xffffffffu : 0u;
        bool full = false;                 // a row's denominator has passed kFull

        for (int k = 0; k < nk; ++k) {
            const uint32_t bar = bars + stage * 8;
            if (k < requested) {
                const bool ok = try_wait(bar, parity) || wait_slow(bar, parity);
                if (!__all_sync(0xffffffffu, ok)) {
                    if (!dead && lane == 0) report_failure(sc.sb, W4A8_ERR_TIMEOUT, kWaitSite);
                    dead = true;
                }
            }
            const uint8_t *slot = ring_ptr + stage * UB;
            // ---- scores ----
            float c[2][NT][4], cs[2][NT][4];
            {
                uint32_t kw[2][2][KW], sat[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint8_t *blk = slot + j * BB;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {            // token g, then token g + 8
                        const uint32_t wk = *reinterpret_cast<const uint32_t *>(blk + 16 * D + 32 * i + 4 * g);
                        const uint32_t off = (wk & 15u) * 0x00400040u + kSixteen;
                        const float f = __low2float(*reinterpret_cast<const __half2 *>(&off));
                        sat[j][i] = sat_constant(off);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            c[j][n][2 * i] = f * qsum[n][0];
                            c[j][n][2 * i + 1] = f * qsum[n][1];
                            cs[j][n][2 * i] = cs[j][n][2 * i + 1] = 0.0f;
                        }
                        const uint8_t *p = blk + (g + 8 * i) * (D / 2) + t * (D / 8);
                        if constexpr (KW == 4) {
                            const uint4 x = *reinterpret_cast<const uint4 *>(p);
                            kw[j][i][0] = x.x; kw[j][i][1] = x.y; kw[j][i][2] = x.z; kw[j][i][3] = x.w;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2 *>(p);
                            kw[j][i][0] = x.x; kw[j][i][1] = x.y;
                        }
                    }
                }
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    uint4 q[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) q[n] = q_frag[n][w][lane];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t e0[4], e1[4];
                        expand(kw[j][0][w], sat[j][0], ek, e0);
                        expand(kw[j][1][w], sat[j][1], ek, e1);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma16(c[j][n], e0[0], e1[0], e0[1], e1[1], q[n].x, q[n].y);
                            mma16(cs[j][n], e0[2], e1[2], e0[3], e1[3], q[n].z, q[n].w);
                        }
                    }
                }
            }
            // wt = the weight's exponent, before the reference is taken off; inv = 1 / step of the value
            float wt[2][NT][4], inv[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint8_t *words = slot + j * BB + 16 * D + 32 * i + 4 * g;
                    const float u = __uint_as_float(*reinterpret_cast<const uint32_t *>(words) & ~15u);
                    const float step = __uint_as_float(*reinterpret_cast<const uint32_t *>(words + 64) & ~15u);
                    const float v = lg2(step);
                    inv[j][i] = rcp(step);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        wt[j][n][2 * i] = fmaf(c[j][n][2 * i] + cs[j][n][2 * i], u * unit[n][0], v);
                        wt[j][n][2 * i + 1] = fmaf(c[j][n][2 * i + 1] + cs[j][n][2 * i + 1], u * unit[n][1], v);
                    }
                }
            const int j0 = (k0 + warp + k * WARPS) * 32;
            if (j0 < lo_max || j0 + 32 > hi_min) {           // some row does not see all of the unit
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = n * 8 + 2 * t + (i & 1), at = j0 + 16 * j + g + (i >> 1) * 8;
                            if (at < row_lo[r] || at >= row_hi[r]) wt[j][n][i] = -INFINITY;
                        }
                    // the words of a token that no row sees are anything (behind the end, in front of the window)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int at = j0 + 16 * j + g + 8 * i;
                        if (at < lo_min || at >= s.len) inv[j][i] = 0.0f;
                    }
                }
            }
            // ---- weights ----
            bool over = full;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float a0 = fmaxf(fmaxf(wt[0][n][0], wt[0][n][2]), fmaxf(wt[1][n][0], wt[1][n][2]));
                const float a1 = fmaxf(fmaxf(wt[0][n][1], wt[0][n][3]), fmaxf(wt[1][n][1], wt[1][n][3]));
                over |= a0 > ref[n][0] + kSlack || a1 > ref[n][1] + kSlack;
            }
            if (__any_sync(0xffffffffu, over)) {
                full = false;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float m = fmaxf(fmaxf(wt[0][n][j], wt[0][n][2 + j]), fmaxf(wt[1][n][j], wt[1][n][2 + j]));
                        if (l[n][j] > kFull) m = fmaxf(m, ref[n][j] + (kShift + kRoom));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                        m = fmaxf(m - kRoom, ref[n][j]);
                        const float keep = ex2(ref[n][j] - m);
                        ref[n][j] = m;
                        l[n][j] *= keep;
                        osum[n][j] *= keep;
#pragma unroll
                        for (int i = 0; i < KT; ++i) {
                            o[n][i][j] *= keep;
                            o[n][i][2 + j] *= keep;
                        }
                    }
            }
            // ---- values ----
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t pb[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float p0 = ex2(wt[j][n][0] - ref[n][0]), p1 = ex2(wt[j][n][1] - ref[n][1]);
                    const float p2 = ex2(wt[j][n][2] - ref[n][0]), p3 = ex2(wt[j][n][3] - ref[n][1]);
                    l[n][0] = fmaf(p2, inv[j][1], fmaf(p0, inv[j][0], l[n][0]));
                    l[n][1] = fmaf(p3, inv[j][1], fmaf(p1, inv[j][0], l[n][1]));
                    pb[n][0] = transpose8(pack_half2(p0, p1));
                    pb[n][1] = transpose8(pack_half2(p2, p3));
                }
                const uint8_t *blk = slot + j * BB;
                const uint2 wva = *reinterpret_cast<const uint2 *>(blk + 16 * D + 64 + 8 * t);
                const uint2 wvb = *reinterpret_cast<const uint2 *>(blk + 16 * D + 64 + 8 * t + 32);
                const uint32_t za = ((wva.y & 15u) * 0x10000u + (wva.x & 15u)) * 0x40u + kSixteen;
                const uint32_t zb = ((wvb.y & 15u) * 0x10000u + (wvb.x & 15u)) * 0x40u + kSixteen;
#pragma unroll
                for (int n = 0; n < NT; ++n) mma16(osum[n], za & only_g0, 0u, zb & only_g0, 0u, pb[n][0], pb[n][1]);
                const uint32_t sa = sat_constant(za), sb = sat_constant(zb);
                constexpr int VW = D / 64;                   // words per token and slice
                const uint8_t *p = blk + 8 * D + g * (D / 2) + t * (D / 8);
                uint32_t xa[2][VW], xb[2][VW];               // [token of the pair][word]
                if constexpr (VW == 2) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(p), y = *reinterpret_cast<const uint4 *>(p + 4 * D);
                    xa[0][0] = x.x; xa[0][1] = x.y; xa[1][0] = x.z; xa[1][1] = x.w;
                    xb[0][0] = y.x; xb[0][1] = y.y; xb[1][0] = y.z; xb[1][1] = y.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(p), y = *reinterpret_cast<const uint2 *>(p + 4 * D);
                    xa[0][0] = x.x; xa[1][0] = x.y;
                    xb[0][0] = y.x; xb[1][0] = y.y;
                }
#pragma unroll
                for (int w = 0; w < VW; ++w)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t ea[4], eb[4];
                        const uint32_t sel = half ? 0x7632u : 0x5410u;
                        expand(perm(xa[0][w], xa[1][w], sel), sa, ek, ea);
                        expand(perm(xb[0][w], xb[1][w], sel), sb, ek, eb);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma16(o[n][4 * w + 2 * half], ea[0], ea[1], eb[0], eb[1], pb[n][0], pb[n][1]);
                            mma16(o[n][4 * w + 2 * half + 1], ea[2], ea[3], eb[2], eb[3], pb[n][0], pb[n][1]);
                        }
                    }
            }
            __syncwarp();                  // every lane is done with the slot
            if (k + S::kStages < nk) {
                request(k + S::kStages, stage);
                if ((k + S::kStages & 15) == 0)              // (every 16 units will do)
#pragma unroll
                    for (int n = 0; n < NT; ++n) full |= l[n][0] > kFull || l[n][1] > kFull;
            }
            if (++stage == S::kStages) {
                stage = 0;
                parity ^= 1u;
            }
        }

        // ---- join the warps: element d of row r of the tile ----
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float v = l[n][j];
                v += __shfl_xor_sync(0xffffffffu, v, 4);
                v += __shfl_xor_sync(0xffffffffu, v, 8);
                v += __shfl_xor_sync(0xffffffffu, v, 16);
                if (g == 0) {              // (the same sum with a higher reference where it is large)
                    const bool large = v > kFull;
                    row_m[warp][n * 8 + 2 * t + j] = large ? ref[n][j] + kLift : ref[n][j];
                    row_l[warp][n * 8 + 2 * t + j] = large ? v * 0x1p-20f : v;
                }
            }
        __syncthreads();                   // also: no warp still reads its ring
        float *join = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = n * 8 + 2 * t + j;
                float m = row_m[0][r];
#pragma unroll
                for (int w = 1; w < WARPS; ++w) m = fmaxf(m, row_m[w][r]);
                const float keep = ex2(ref[n][j] - m);
                const float sum = __shfl_sync(0xffffffffu, osum[n][j], t);
                float *to = join + ((size_t)warp * R + r) * S::kPad + g * (D / 8);
#pragma unroll
                for (int i = 0; i < KT; ++i)
                    *reinterpret_cast<float2 *>(to + 2 * i) =
                        make_float2(fmaf(-2.0f, o[n][i][j], -sum) * keep, fmaf(-2.0f, o[n][i][2 + j], -sum) * keep);
            }
        if (tid < R) {
            float m = row_m[0][tid], v = 0.0f;
#pragma unroll
            for (int w = 1; w < WARPS; ++w) m = fmaxf(m, row_m[w][tid]);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += row_l[w][tid] * ex2(row_m[w][tid] - m);
            tile_m[tid] = m;
            tile_l[tid] = v;
        }
        __syncthreads();
        const int part_size = R * (D + 2);
        constexpr int kQuads = R * D / 4;
        auto write_row = [&](int r, int d, float4 v, float m, float lsum) {
            const int i = sc.group.div(tile * R + r);
            const size_t at = ((size_t)(s.row0 + i) * a.q_heads + h * group + tile * R + r - i * group) * D + d;
            const float inv = lsum > 0.0f ? __fdiv_rn(1.0f, lsum) : 0.0f;
            v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
            uint2 out;
            if (a.o_bf16) {
                const float top = __uint_as_float(0x7f7f0000u);
                const __nv_bfloat162 x = __floats2bfloat162_rn(fminf(fmaxf(v.x, -top), top), fminf(fmaxf(v.y, -top), top));
                const __nv_bfloat162 y = __floats2bfloat162_rn(fminf(fmaxf(v.z, -top), top), fminf(fmaxf(v.w, -top), top));
                out.x = *reinterpret_cast<const uint32_t *>(&x);
                out.y = *reinterpret_cast<const uint32_t *>(&y);
            } else {
                const float top = 65504.0f;
                out.x = pack_half2(fminf(fmaxf(v.x, -top), top), fminf(fmaxf(v.y, -top), top));
                out.y = pack_half2(fminf(fmaxf(v.z, -top), top), fminf(fmaxf(v.w, -top), top));
            }
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.O) + at) = out;
            if (a.lse && d == 0) a.lse[at / D] = lsum > 0.0f ? (m + lg2(lsum)) * kLn2 : -INFINITY;
        };
        float *part = sc.partials + ((size_t)blockIdx.x * 2 + (first_unit <= begin ? 0 : 1)) * part_size;
        for (int i = tid; i < kQuads; i += THREADS) {
            const int r = i / (D / 4), d = (i % (D / 4)) * 4;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(join + ((size_t)w * R + r) * S::kPad + d);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            if (!whole) __stcg(reinterpret_cast<float4 *>(part + 2 * R) + i, v);
            else if (r < rows_here) write_row(r, d, v, tile_m[r], tile_l[r]);
        }
        if (!whole) {
            if (tid < R) {
                __stcg(part + tid, tile_m[tid]);
                __stcg(part + R + tid, tile_l[tid]);
            }
            __syncthreads();
            const int w0 = (int)quotient(first_unit, per), w1 = (int)quotient(first_unit + item_units - 1, per);
            if (tid == 0) {                // releases what the CTA has stored, acquires the parts of those before it
                int before;
                asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(sc.counters + w0) : "memory");
                last_part = before == w1 - w0;
            }
            __syncthreads();
            if (last_part) {
                // part of worker w: its first segment, unless the item begins inside its share.  A warp takes every
                // WARPS-th part, all of their loads in flight together; the warps' sums are joined as above.
                const bool inside = first_unit > (long long)w0 * per;
                const float *rest = sc.partials + (size_t)w0 * 2 * part_size;
                const int parts = w1 - w0 + 1;
                auto part_of = [&](int p) { return rest + (p > 0 ? (size_t)p * 2 * part_size : inside ? (size_t)part_size : 0); };
                float m = kNoReference, lsum = 0.0f;         // of row lane % R
#pragma unroll 8
                for (int p = warp; p < parts; p += WARPS) m = fmaxf(m, __ldcg(part_of(p) + lane % R));
                constexpr int kMine = kQuads / 32;           // quad lane + 32 k: row 32 k / (D / 4) + lane / (D / 4)
                float4 v[kMine];
#pragma unroll
                for (int k = 0; k < kMine; ++k) v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
                for (int p = warp; p < parts; p += WARPS) {
                    const float *x = part_of(p);
                    const float keep = ex2(__ldcg(x + lane % R) - m);
                    lsum = fmaf(__ldcg(x + R + lane % R), keep, lsum);
#pragma unroll
                    for (int k = 0; k < kMine; ++k) {
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(x + 2 * R) + lane + 32 * k);
                        const float f = __shfl_sync(0xffffffffu, keep, (lane + 32 * k) / (D / 4));
                        v[k].x = fmaf(y.x, f, v[k].x);
                        v[k].y = fmaf(y.y, f, v[k].y);
                        v[k].z = fmaf(y.z, f, v[k].z);
                        v[k].w = fmaf(y.w, f, v[k].w);
                    }
                }
                if (lane < R) {
                    row_m[warp][lane] = m;
                    row_l[warp][lane] = lsum;
                }
#pragma unroll
                for (int k = 0; k < kMine; ++k) {
                    const int i = lane + 32 * k;
                    *reinterpret_cast<float4 *>(join + ((size_t)warp * R + i / (D / 4)) * S::kPad + i % (D / 4) * 4) = v[k];
                }
                __syncthreads();
                for (int i = tid; i < kQuads; i += THREADS) {
                    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
                    if (r >= rows_here) continue;
                    float top = row_m[0][r], den = 0.0f;
#pragma unroll
                    for (int w = 1; w < WARPS; ++w) top = fmaxf(top, row_m[w][r]);
                    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < WARPS; ++w) {
                        const float keep = ex2(row_m[w][r] - top);
                        const float4 x = *reinterpret_cast<const float4 *>(join + ((size_t)w * R + r) * S::kPad + d);
                        den = fmaf(row_l[w][r], keep, den);
                        y.x = fmaf(x.x, keep, y.x);
                        y.y = fmaf(x.y, keep, y.y);
                        y.z = fmaf(x.z, keep, y.z);
                        y.w = fmaf(x.w, keep, y.w);
                    }
                    write_row(r, d, y, top, den);
                }
                if (tid == 0) sc.counters[w0] = 0;           // ready for the next call
            }
        }
        // the join buffer was written by ordinary stores: order them before the next copies into the ring
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
}

// Rows per tile and warps per CTA.
struct Variant {
    int nt, warps, ctas;
};
Variant pick(const KvAttnArgs &a, int sms)
{
    const int group = a.q_heads / a.cache.heads;
    const long long rows = (long long)group * ((a.batch.rows + a.batch.batch - 1) / a.batch.batch);
    Variant v;
    v.nt = rows > 8 ? 2 : 1;
    const long long items = (long long)a.batch.batch * a.cache.heads * ((rows + 8 * v.nt - 1) / (8 * v.nt));
    // few items: every item is split over several CTAs, and wide CTAs leave fewer parts to join (one sequence of
    // 131001 tokens, 8 heads: 52.6 us wide, 56.2 us narrow); many: narrow CTAs, whose ends and beginnings overlap
    // with their neighbours' streaming (64 ragged sequences of 8 heads: 84.9 us wide, 79.7 us narrow)
    const int per_sm = v.nt == 1 ? 16 : 12;
    v.warps = items >= sms ? 4 : per_sm / 2;
    v.ctas = sms * (per_sm / v.warps);
    return v;
}

// Which kernel, by the query rows that share a key head, on average over the sequences.  The prefill kernel's
// tile is 256 rows and costs about the same from one row on; the decode kernel's cost grows with every 16.
// Measured in us, decode / prefill, 8 key heads of 128: 4 sequences of 3000 tokens, 32 rows 25 / 37,
// 64 rows 35 / 37, 96 rows 49 / 37; 16 of 3000, 64 rows 92 / 86, 128 rows 171 / 91; one of 32000,
// 64 rows 64 / 73, 96 rows 98 / 74.  With little work the decode kernel stays ahead further (one of 4000, 128
// rows 35 / 35; one of 500, 128 rows 17 / 22), but the lengths are known on the device only.
bool use_prefill(int rows, int batch, int q_heads, int kv_heads)
{
    return (long long)(q_heads / kv_heads) * rows > 64ll * batch;
}

template <int D, int NT, int WARPS>
cudaError_t launch(const KvAttnArgs &a, const Schedule &sc, int ctas, cudaStream_t st)
{
    using S = Shape<D, NT, WARPS>;
    static std::atomic<int> raised[kMaxDevices];
    const cudaError_t e = raise_smem_limit(kv_decode_kernel<D, NT, WARPS>, S::kSmem, raised);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kv_decode_kernel<D, NT, WARPS>, dim3(ctas), dim3(WARPS * 32), S::kSmem, st, a, sc);
}
template <int D>
cudaError_t launch(const KvAttnArgs &a, const Schedule &sc, const Variant &v, cudaStream_t st)
{
    if (v.nt == 1) return v.warps == 4 ? launch<D, 1, 4>(a, sc, v.ctas, st) : launch<D, 1, 8>(a, sc, v.ctas, st);
    return v.warps == 4 ? launch<D, 2, 4>(a, sc, v.ctas, st) : launch<D, 2, 6>(a, sc, v.ctas, st);
}

}  // namespace

// Status block, counters, and two partial results per CTA (at most 4 CTAs with one tile of eight rows or
// 3 with two per SM).
size_t kv_attention_workspace(int rows, int batch, int q_heads, int kv_heads, int D)
{
    if (use_prefill(rows, batch, q_heads, kv_heads)) return kv_prefill_workspace(D);
    const int sms = device_sms();
    return sizeof(StatusBlock) + kv_counters_bytes(sms) + (size_t)sms * 3 * 2 * 16 * (D + 2) * sizeof(float);
}

cudaError_t launch_kv_attention(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st)
{
    if (use_prefill(a.batch.rows, a.batch.batch, a.q_heads, a.cache.heads)) return launch_kv_prefill(a, workspace, st);
    const int sms = device_sms();
    const Variant v = pick(a, sms);
    const Schedule sc = {reinterpret_cast<StatusBlock *>(workspace), reinterpret_cast<int *>(workspace + sizeof(StatusBlock)),
                         reinterpret_cast<float *>(workspace + sizeof(StatusBlock) + kv_counters_bytes(sms)), v.warps, kLead,
                         Divisor((uint32_t)(a.q_heads / a.cache.heads))};
    return a.cache.D == 64 ? launch<64>(a, sc, v, st) : launch<128>(a, sc, v, st);
}

}  // namespace w4a8
