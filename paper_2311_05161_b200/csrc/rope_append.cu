// Rotary positions on queries and keys, and the rows' keys and values into the 4-bit cache, in one pass.
//
// A pair (a, b) of a vector's elements is turned by the angle position * inv_freq:
//   a' = a cos - b sin,  b' = b cos + a sin   (binary32, one rounding per operation),
// Q is rounded once to its 16-bit type, K goes into the quantizer of the cache as it is.  The angle is a product in binary64
// (exact up to positions of 2^29), its fraction of a turn is taken there with 1 / (2 pi) in two parts, and sine and
// cosine come from binary64 and are rounded once: a far position loses nothing, where a binary32 product is off by
// a sixteenth of a radian at 10^6.
//
// The work is a list of units, four vectors (keys, values or queries) of as many rows as fit a warp side by side, D/8 lanes to a
// vector.  The warps of one wave of CTAs share the list evenly by what the units cost, and a warp loads a unit's
// vectors while it works on the one before.  Entering a row it computes the row's sines and cosines into shared memory, for all its
// heads.  Where a vector is turned, a lane has four whole pairs (for halves: elements 4 l .. 4 l + 3 and their partners half a
// rotation further on, so that no element changes lanes), else eight consecutive elements.  The four vectors of a unit are
// quantized together: their ranges are reduced side by side, so that a lane is left with one vector's and the two
// divisions of a step are done once for four.
//
// Four prompts (10348 rows, 32 query and 8 key heads of 128, 223 MB): 48.0 us, 4.6 TB/s, 0.71 of the copy rate; issue slots 62 %
// busy, and the same walk without sines, quantizer and cache stores still takes 45 us.  Measured and left: a row's vectors
// split over CTAs, with a lane's partner elements by shuffles 53.9 us; rows in CTAs with barriers 54.7; asynchronous copies into
// shared memory instead of registers 52.4; packed binary32 products 52.7; 5 or 6 CTAs per SM (fewer registers) 50.6 and
// 53.5; stores that stay in L2 54.0.  Eight rows: 3.2 us, a launch and the chain of slot, position, sine, range and code.
#include <type_traits>

#include "kv_cache.cuh"

namespace w4a8 {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32, kCtas = 4;

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

// Eight values rounded once to 16 bits, those beyond the type's range to its largest finite ones (they are rare: one
// look at the largest of eight).
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> __device__ __forceinline__ float largest();
template <> __device__ __forceinline__ float largest<__half>() { return 65504.0f; }
template <> __device__ __forceinline__ float largest<__nv_bfloat16>() { return __uint_as_float(0x7f7f0000u); }
template <typename T>
__device__ __forceinline__ void hold_in_range(float (&x)[8])
{
    float top = fabsf(x[0]);
#pragma unroll
    for (int k = 1; k < 7; k += 2) top = max3(top, fabsf(x[k]), fabsf(x[k + 1]));
    if (fmaxf(top, fabsf(x[7])) > largest<T>()) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = fminf(fmaxf(x[k], -largest<T>()), largest<T>());
    }
}

// What the units of a row group cost beside one another (instructions, roughly), for even shares.
constexpr int kKeyCost = 6, kValueCost = 5, kQueryCost = 2;
struct Units {
    int kv, q;                               // units of the keys (and of the values), of the queries
    __host__ __device__ int all() const { return 2 * kv + q; }
    __host__ __device__ int row_cost() const { return kv * (kKeyCost + kValueCost) + q * kQueryCost; }
    // the first unit that begins at `cost` or behind it
    __device__ int from(int cost) const
    {
        if (cost <= kv * kKeyCost) return (cost + kKeyCost - 1) / kKeyCost;
        cost -= kv * kKeyCost;
        if (cost <= kv * kValueCost) return kv + (cost + kValueCost - 1) / kValueCost;
        return 2 * kv + (cost - kv * kValueCost + kQueryCost - 1) / kQueryCost;
    }
};

// UNIT: vectors of a unit, 4 or 1.
template <typename T, int D, bool INTERLEAVED, int UNIT>
__global__ void __launch_bounds__(kThreads, kCtas)
rope_append_kernel(const RopeArgs a, const KvCache c, const Units units, StatusBlock *sb)
{
    constexpr int LPV = D / 8, GROUPS = 32 / LPV;              // lanes of a vector, rows of a row group
    __shared__ __align__(16) float all_turns[kWarps][GROUPS][2][D / 2];    // cosines, sines
    allow_dependents();
    dependent_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LPV;
    float (*turns)[2][D / 2] = all_turns[warp];
    const int half = a.rotary / 2, row_cost = units.row_cost();
    const long long all_slots = (long long)c.num_pages << c.page_shift;
    const bool turned = 8 * l < a.rotary;
    // this lane's first four elements of a turned vector, and its others
    const int e0 = INTERLEAVED || !turned ? 8 * l : 4 * l, e1 = INTERLEAVED || !turned ? 8 * l + 4 : half + 4 * l;
    const size_t head_bytes = ((size_t)1 << c.page_shift) * (D + 8);
    const int n_units = units.all();
    // ---- this warp's share: from unit u of row group `group` to unit last_u of row group last_group, without that one ----
    const uint32_t share = blockIdx.x * kWarps + warp, shares = gridDim.x * kWarps, row_groups = (a.rows + GROUPS - 1) / GROUPS;
    int group, u, last_group, last_u;
    auto step = [&](int &g, int &v) {
        if (++v == n_units) ++g, v = 0;
    };
    if constexpr (UNIT == 1) {               // a unit for every warp, and warps without one
        last_group = group = (int)(share / n_units);
        last_u = u = (int)(share - group * n_units);
        if ((uint32_t)group >= row_groups) return;
        step(last_group, last_u);
    } else {                                 // the units that begin in an even part of the list's cost
        const unsigned long long total = (unsigned long long)row_groups * row_cost;
        auto place = [&](uint32_t part, int &g, int &v) {
            const unsigned long long cost = total * part / shares;
            g = (int)(cost / row_cost);
            v = units.from((int)(cost - (unsigned long long)g * row_cost));
            if (v == n_units) ++g, v = 0;
        };
        place(share, group, u);
        place(share + 1, last_group, last_u);
    }
    auto kind_of = [&](int v) { return v < units.kv ? 0 : v < 2 * units.kv ? 1 : 2; };         // keys, values, queries
    auto before = [&](int g, int v) { return g < last_group || (g == last_group && v < last_u); };
    struct Raw {
        uint2 v[UNIT][2];
    };
    // (Places without a vector keep what they hold: nothing of it is stored.)
    auto load = [&](int at_group, int v, Raw &raw) {
        const int kind = kind_of(v), h0 = (v - kind * units.kv) * UNIT, r = at_group * GROUPS + lane / LPV;
        const int n = r < a.rows ? (kind == 2 ? a.q_heads : c.heads) - h0 : 0;
        const T *from = kind == 0 ? static_cast<const T *>(a.K) : kind == 1 ? static_cast<const T *>(a.V) : static_cast<const T *>(a.Q);
        from += (size_t)r * (kind == 0 ? a.k_stride : kind == 1 ? a.v_stride : a.q_stride) + (size_t)h0 * D;
        const T *p0 = from + (kind == 1 ? 8 * l : e0), *p1 = from + (kind == 1 ? 8 * l + 4 : e1);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            if (j < n) {
                raw.v[j][0] = __ldcs(reinterpret_cast<const uint2 *>(p0 + j * D));
                raw.v[j][1] = __ldcs(reinterpret_cast<const uint2 *>(p1 + j * D));
            }
        }
    };
    bool here = false;                       // this lane's row has a slot (lanes without one take part in the shuffles)
    int s = 0;                               // its place in its block
    uint8_t *block = c.pages;                // of head 0
    int row = 0;
    auto enter = [&](int at_group) {         // a new row group: slots, sines and cosines
        row = at_group * GROUPS + lane / LPV;
        long long slot = row < a.rows ? __ldca(reinterpret_cast<const long long *>(a.slots) + row) : -1;
        if (slot >= all_slots) {
            if (l == 0) report_failure(sb, W4A8_ERR_BAD_TABLE, row);
            slot = -1;
        }
        here = slot >= 0;
        if (here) {
            const int in_page = (int)(slot & ((1ll << c.page_shift) - 1));
            s = in_page & 15;
            block = c.pages + (size_t)(slot >> c.page_shift) * c.page_bytes() + (size_t)(in_page >> 4) * kv_block_bytes(D);
        }
        __syncwarp();                        // the turns of the group before are no longer needed
#pragma unroll
        for (int k0 = 0; k0 < D / 2; k0 += LPV) {              // four pairs of the row
            const int k = k0 + l;
            if (row >= a.rows || k >= half) break;
            int axis = a.pair_axis ? __ldca(a.pair_axis + k) : 0;
            if ((unsigned)axis >= (unsigned)a.axes) {
                report_failure(sb, W4A8_ERR_BAD_TABLE, row);
                axis = 0;
            }
            float *t = &turns[lane / LPV][0][k];
            turn(__ldca(a.positions + (size_t)axis * a.rows + row), __ldca(a.inv_freq + k), t[D / 2], t[0]);
        }
        __syncwarp();
    };
    // the eight elements of a vector: e0 .., e1 ..
    auto elements = [&](const uint2 (&v)[2], float (&x)[8]) {
        const float2 f[4] = {to_float2<T>(v[0].x), to_float2<T>(v[0].y), to_float2<T>(v[1].x), to_float2<T>(v[1].y)};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = f[k].x;
            x[2 * k + 1] = f[k].y;
        }
    };
    auto rotate = [&](float (&x)[8], const float4 &cs, const float4 &sn) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int m = INTERLEAVED ? 2 * k : k, o = INTERLEAVED ? 2 * k + 1 : k + 4;
            const float p0 = x[m], p1 = x[o], co = (&cs.x)[k], si = (&sn.x)[k];
            x[m] = __fsub_rn(__fmul_rn(p0, co), __fmul_rn(p1, si));
            x[o] = __fadd_rn(__fmul_rn(p1, co), __fmul_rn(p0, si));
        }
    };
    auto queries = [&](int h0, const Raw &raw) {
        if (!here) return;
        const float4 cs = *reinterpret_cast<const float4 *>(&turns[lane / LPV][0][4 * l % (D / 2)]);
        const float4 sn = *reinterpret_cast<const float4 *>(&turns[lane / LPV][1][4 * l % (D / 2)]);
        T *to = static_cast<T *>(a.Q_out) + (size_t)row * a.q_out_stride + (size_t)h0 * D;
        const int n = a.q_heads - h0;
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            if (j >= n) break;
            float x[8];
            elements(raw.v[j], x);
            if (turned) {
                rotate(x, cs, sn);
                hold_in_range<T>(x);
            }
            __stcs(reinterpret_cast<uint2 *>(to + j * D + e0), make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])));
            __stcs(reinterpret_cast<uint2 *>(to + j * D + e1), make_uint2(pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])));
        }
    };
    auto quantize = [&](auto is_value, int h0, const Raw &raw) {
        constexpr bool VALUE = decltype(is_value)::value;
        float x[UNIT][8], lo[UNIT], hi[UNIT];
        if constexpr (VALUE) {
#pragma unroll
            for (int j = 0; j < UNIT; ++j) elements(raw.v[j], x[j]);
        } else {
            const float4 cs = *reinterpret_cast<const float4 *>(&turns[lane / LPV][0][4 * l % (D / 2)]);
            const float4 sn = *reinterpret_cast<const float4 *>(&turns[lane / LPV][1][4 * l % (D / 2)]);
#pragma unroll
            for (int j = 0; j < UNIT; ++j) {
                elements(raw.v[j], x[j]);
                if (turned && here) rotate(x[j], cs, sn);
            }
        }
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            lo[j] = hi[j] = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                lo[j] = min3(lo[j], x[j][k], x[j][k + 1]);
                hi[j] = max3(hi[j], x[j][k], x[j][k + 1]);
            }
        }
        float my_r;
        int my_z;
        uint32_t my_word;
        if constexpr (UNIT == 4) my_word = kv_four_words<LPV>(lo, hi, lane, my_r, my_z);
        else {
#pragma unroll
            for (int o = LPV / 2; o > 0; o >>= 1) {
                lo[0] = fminf(lo[0], __shfl_xor_sync(0xffffffffu, lo[0], o));
                hi[0] = fmaxf(hi[0], __shfl_xor_sync(0xffffffffu, hi[0], o));
            }
            my_word = kv_range_word(lo[0], hi[0], my_r, my_z);
        }
        const uint32_t my_zz = kv_twice(my_z);
        // four elements' codes are two bytes; the places of this lane's two halves
        const int a0 = VALUE ? 8 * l : e0, a1 = VALUE ? 8 * l + 4 : e1;
        uint8_t *to = block + h0 * head_bytes;
        const int n = c.heads - h0;
        {                                    // the words, by one lane each
            constexpr int OWN = LPV / UNIT;
            const int j = UNIT == 1 ? 0 : (l / OWN & 1) + (l / OWN & 2);
            if (l % OWN == 0 && here && j < n) *reinterpret_cast<uint32_t *>(to + j * head_bytes + kv_word_offset(D, VALUE, s)) = my_word;
        }
        uint8_t *to0 = to + kv_code_offset(D, VALUE, s, a0 / 8) + (a0 & 4) / 2, *to1 = to + kv_code_offset(D, VALUE, s, a1 / 8) + (a1 & 4) / 2;
#pragma unroll
        for (int j = 0; j < UNIT; ++j) {
            uint32_t zz = my_zz;
            float r_step = my_r;
            if constexpr (UNIT == 4) {
                zz = __shfl_sync(0xffffffffu, my_zz, kv_owner_of<LPV>(j), LPV);
                r_step = __shfl_sync(0xffffffffu, my_r, kv_owner_of<LPV>(j), LPV);
            }
            if (here && j < n) {
                const uint32_t codes = kv_code_word(x[j], r_step, zz);
                if (VALUE || INTERLEAVED || !turned) *reinterpret_cast<uint32_t *>(to0) = codes;
                else {
                    *reinterpret_cast<uint16_t *>(to0) = (uint16_t)codes;
                    *reinterpret_cast<uint16_t *>(to1) = (uint16_t)(codes >> 16);
                }
            }
            to0 += head_bytes;
            to1 += head_bytes;
        }
    };
    if (!before(group, u)) return;
    int entered = -1;
    auto work = [&](const Raw &raw) {
        if (group != entered) enter(entered = group);
        const int kind = kind_of(u), h0 = (u - kind * units.kv) * UNIT;
        if (kind == 0) quantize(std::false_type(), h0, raw);
        else if (kind == 1) quantize(std::true_type(), h0, raw);
        else queries(h0, raw);
    };
    Raw raw;
    load(group, u, raw);
    for (;;) {
        int next_group = group, next_u = u;
        step(next_group, next_u);
        const bool more = before(next_group, next_u);
        Raw next;
        if (more) load(next_group, next_u, next);
        work(raw);
        if (!more) return;
        raw = next;
        group = next_group;
        u = next_u;
    }
}

template <typename T, int D, int UNIT>
cudaError_t launch(const RopeArgs &a, int interleaved, const KvCache &c, const Units &units, long long all, StatusBlock *sb, cudaStream_t st)
{
    // one wave of CTAs whose warps have even shares; fewer where there are fewer units than warps
    const long long ctas = (all + kWarps - 1) / kWarps, most = (long long)kCtas * device_sms();
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    return interleaved ? launch_overlapped(rope_append_kernel<T, D, true, UNIT>, grid, dim3(kThreads), 0, st, a, c, units, sb)
                       : launch_overlapped(rope_append_kernel<T, D, false, UNIT>, grid, dim3(kThreads), 0, st, a, c, units, sb);
}
template <typename T, int D>
cudaError_t launch(const RopeArgs &a, int interleaved, const KvCache &c, StatusBlock *sb, cudaStream_t st)
{
    const int groups = 256 / D;
    const long long row_groups = (a.rows + groups - 1) / groups;
    // Units of single vectors as long as every warp has one of them at most: the time is then a vector's chain of steps.
    const Units one = {c.heads, a.q_heads}, four = {(c.heads + 3) / 4, (a.q_heads + 3) / 4};
    return row_groups * one.all() <= (long long)kCtas * device_sms() * kWarps
               ? launch<T, D, 1>(a, interleaved, c, one, row_groups * one.all(), sb, st)
               : launch<T, D, 4>(a, interleaved, c, four, row_groups * four.all(), sb, st);
}

}  // namespace

cudaError_t launch_rope_kv_append(const RopeArgs &a, int bf16, int interleaved, const KvCache &c, StatusBlock *sb,
                                  cudaStream_t st)
{
    if (c.D == 64) return bf16 ? launch<__nv_bfloat16, 64>(a, interleaved, c, sb, st) : launch<__half, 64>(a, interleaved, c, sb, st);
    return bf16 ? launch<__nv_bfloat16, 128>(a, interleaved, c, sb, st) : launch<__half, 128>(a, interleaved, c, sb, st);
}

}  // namespace w4a8
