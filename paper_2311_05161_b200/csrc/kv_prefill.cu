// Attention over the 4-bit cache, prefill form: many query rows per sequence.
//
// A CTA works on 256 query rows (the heads that share a key head, times tokens) as two tiles of 128, and
// walks over the keys in units of 64 tokens.  Both products run on the tensor cores with the accumulators
// in tensor memory: S = Q K^T (tcgen05 kind::f16, operands in shared memory) and O += P V with P read
// from tensor memory, where it takes the place of its scores.  Tensor memory is full: two score buffers of 64
// columns and an output tile of 128 per row tile.  Two buffers, so that the scores of the next unit are
// computed while the softmax of this one runs (units of 128 tokens with one buffer left every row tile with
// a chain of softmax and MMAs: 173 against 159 us on the 1024-row chunk below).
//
// Roles: eight softmax warps, a thread per row; eight expanding warps, four threads per token, which turn a unit's
// codes into binary16 operand tiles in shared memory (four units of keys and values); two
// warps issue the MMAs, one for each row tile (a thread issues an MMA per 100 cycles or so beside the busy
// softmax warps, twice what the MMAs take); one lists the pieces of work.  Twenty warps in all.
// Every hand-over is an mbarrier with a bounded wait; a wait that runs out raises a flag that ends all roles.
//
// Numbers: both operands are exact levels (times -1/2).  A token's key step multiplies its score column; its value
// step enters the weight's exponent, as in the decode form, so that the weights' rounding to binary16 is the
// only one.  A thread looks over its row's scores for their maximum first; where a weight would exceed 2^15
// against the running reference, it moves the reference and scales the output row in tensor memory.  (One
// pass that computed the weights at once and again after an overflow was slower: on scores that spread
// over five bits one unit in eight overflowed in some row of a warp.)
//
// Bounds per unit and SM for D = 128: 1024 cycles of MMA (a 128 x 64 x 128 and a 128 x 128 x 64 product per row
// tile), 1024 cycles of exponentials at 16 per cycle, about 500 cycles of packed binary16 arithmetic to
// expand 16384 codes: the expansion is shared by 256 rows, which is why the two tiles are one CTA's.
// Measured: the last 1024 of 4096 tokens (8 key heads, 32 query heads of 128) 109 us, 553 TFLOP/s, tensor
// pipe 28 %, issue slots 56 % busy; 4 prompts of 2048: 285 us.  From runs of several lengths (items of 256 rows, one or
// more per CTA): 1.47 us per unit (2890 cycles at 1965 MHz; D = 64: 1.34 us), 17 us for the launch and a CTA's first
// piece, 10 to 13 us for each further piece.  A unit's time is the softmax's chain of wait, load, maximum, exponentials and
// store.  A piece's is what does not overlap between pieces: queries (4 us to their common maximum, 1.5 us to the operand
// tile), first keys, output or parts (2.7 us).  The chunk is 49 units
// and 1.9 pieces per CTA, the prompts 114 units and 7.9 pieces: a quarter and two fifths of the time lie
// outside the units.  (Sixteen softmax warps, two threads per row, were slower for their exchange of maxima: 120 us.)
// Leaving out exponentials, token constants, expansion and moved references all together takes 13 us off the chunk, three of four
// MMAs 8 us: no pipe is a unit's time, the hand-overs are.
//
// The extended forms (kSinks, kTree) take their units from the sinks and then from the window, and mask a unit that some row does not
// see whole by 64 bits per row, made from bounds and the row's tree mask.  A chunk of 1024 rows at 9000, window 4096, 4 sinks: 122 us
// (120.9 without the sinks in the plain form); 16 trees of 40 to 64 nodes, 32 / 8 heads, 1000 to 6000 tokens: 124 us (causal
// rows in the plain form 122.5).
#include "kv_attention.cuh"

namespace w4a8 {

namespace {

constexpr int kRows = 256, kUnit = 64, kUnitShift = 6;
constexpr int kSoftmaxWarps = 8, kExpandWarps = 8, kMmaWarp = kSoftmaxWarps + kExpandWarps, kListWarp = kMmaWarp + 2;
constexpr int kWarps = 20, kThreads = 32 * kWarps;         // the last one only helps to find the share
constexpr int kRing = 4;                                   // units of expanded keys, and of values
constexpr int kConstSlots = 8;                             // more than kRing: a slot is rewritten after its unit's softmax
constexpr int kLead = 6;                                   // an item's fixed cost, in units
// What a CTA loses where its share is parts of two items instead of one item, in units: a second piece and the join; and where it is a part
// of one, as with fewer items than half the CTAs: the join alone.  In us, 4 sinks, items of head dimension 128 one by one / in even shares: 128
// items of 73 places (units and lead, window 4096) 122.0 / 124.9, of 9 to 48 places 21.7 / 28.7 to 79.3 / 85.0; 64 items of 10 places 22.9 / 23.5, of 12
// 25.4 / 26.0, of 16 29.8 / 29.6; 48 of 12 25.1 / 24.4, of 15 29.0 / 26.2; 2 to 32 items of 9 places 20.3 / 21.8, of 10 22.1 / 23.5, of 12 24.3 / 21.7.
constexpr int kTwoParts = 10, kOnePart = 6;
constexpr int kWaitSite = 950;
constexpr int kApart = 16;                                 // a row at most 2^16 below its tile's largest is good to 2^-23 of its own largest element

// -------------------------------------------------------------------- tensor core wrappers
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operand descriptors: rows of 128 bytes (64 elements) in 128-byte swizzle, eight rows 1024 bytes apart; the second
// 64 elements of a row lie one tile of rows further on.  As a K-major operand (queries, keys) a row is
// an index of M or N; as an MN-major one (values) a row is an index of K and the tiles follow each other
// along N (leading-dimension offset).  The high word is the same for all; the low one holds address and
// leading-dimension offset in units of 16 bytes.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t leading)
{
    return ((addr & 0x3FFFFu) >> 4) | ((leading >> 4) << 16);
}
// D += A B with A in shared memory / in tensor memory, binary16 operands, binary32 accumulator.  (Two 32-bit words
// per descriptor: a role with few registers issues these.)
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi)
                 : "memory");
}
__device__ __forceinline__ void tmem_request32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
// All loads so far have arrived; the registers pass through, so that nothing reads them before.
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                   "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                   "+r"(r[28]), "+r"(r[29])
                 :
                 : "memory");
    asm volatile("" : "+r"(r[30]), "+r"(r[31])::"memory");
}
// 64 columns of this thread's lane.
__device__ __forceinline__ void tmem_load64(uint32_t addr, float (&r)[64])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
          "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
          "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31]),
          "=f"(r[32]), "=f"(r[33]), "=f"(r[34]), "=f"(r[35]), "=f"(r[36]), "=f"(r[37]), "=f"(r[38]), "=f"(r[39]),
          "=f"(r[40]), "=f"(r[41]), "=f"(r[42]), "=f"(r[43]), "=f"(r[44]), "=f"(r[45]), "=f"(r[46]), "=f"(r[47]),
          "=f"(r[48]), "=f"(r[49]), "=f"(r[50]), "=f"(r[51]), "=f"(r[52]), "=f"(r[53]), "=f"(r[54]), "=f"(r[55]),
          "=f"(r[56]), "=f"(r[57]), "=f"(r[58]), "=f"(r[59]), "=f"(r[60]), "=f"(r[61]), "=f"(r[62]), "=f"(r[63])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ float4 load_shared4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32])
{
    tmem_request32(addr, r);
    tmem_arrived(r);
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Instruction descriptor: binary16 A and B, binary32 D, M = 128; B of the value product is MN-major.
__host__ __device__ constexpr uint32_t instr_desc(int n, int b_mn_major)
{
    return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
template <int D>
struct Layout {
    static constexpr int kHalves = D / 64;                 // 64-element parts of a row
    static constexpr int kQPart = 128 * 128, kQTile = kHalves * kQPart;          // 128 query rows
    static constexpr int kPartBytes = kUnit * 128, kTile = kHalves * kPartBytes; // a unit's keys or values
    static constexpr int kOffK = 2 * kQTile, kOffV = kOffK + kRing * kTile;
    static constexpr int kOffConst = kOffV + kRing * kTile;
    static constexpr int kConstBytes = kUnit * 12;         // per token: key step * unit; log2 of the value step; its inverse
    static constexpr int kOffQmax = kOffConst + kConstSlots * kConstBytes;
    static constexpr int kOffRowScale = kOffQmax + 2 * kSoftmaxWarps * 4;        // per row, see the queries
    static constexpr int kOffBars = kOffRowScale + kRows * 4;
    // barriers
    static constexpr int kKFull = 0, kKEmpty = kKFull + kRing, kVFull = kKEmpty + kRing, kVEmpty = kVFull + kRing,
                         kSFull = kVEmpty + kRing, kPReady = kSFull + 4, kODone = kPReady + 4,
                         kQFull = kODone + 4, kQmax = kQFull + 2, kDrain = kQmax + 1, kPieceFull = kDrain + 2,
                         kPieceEmpty = kPieceFull + 2, kBars = kPieceEmpty + 2;
    static constexpr int kSmem = kOffBars + kBars * 8 + 1024;
    static_assert(kSmem + 1024 <= 232448, "shared memory of an SM");
};

struct Schedule {
    StatusBlock *sb;
    float *partials;           // [workers][2] parts of 256 * (D + 2) numbers
    struct Shared *shared;     // [workers]
    Divisor group;
};

// The item that begins in a CTA's share and ends in a later one's, for the kernel that joins its parts.
struct Shared {
    int parts;                                 // 0: there is none
    int inside;                                // it does not begin with the share
    int row0, h, tile, rows;
    int pad[2];
};

// A piece of an item that falls into a CTA's share, as the scheduling warp hands it to the others.
struct Piece {
    int b, h, tile, rows;                      // sequence, key head, row tile, its rows
    int row0, n, len;                          // of the sequence
    int unit0, count;                          // units to walk; count < 0: no more pieces
    int lo;                                    // first token that a row of the tile sees
    int few, few0;                             // the extended form: its first `few` units hold sinks and lie from few0 on
    int whole;                                 // the item lies in this share alone
    int slot;                                  // else: where the part goes
};

struct Control {
    volatile int abort;
    uint32_t tmem;
    int found_b, found_tile;
    long long found_off;
    long long warp_len[kWarps];
    int warp_items[kWarps], warp_longest[kWarps];
    Piece piece[2];
};

__device__ bool wait_long(uint32_t bar, uint32_t parity, Control *ctl, StatusBlock *sb, int where, int pause)
{
    unsigned long long t0 = 0, t;
    for (uint32_t i = 1;; ++i) {
        if (pause) __nanosleep(pause);
        if (try_wait(bar, parity)) return true;
        if ((i & 63u) == 0u) {
            if (ctl->abort) return false;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            else if (t - t0 > kWaitNs) {
                ctl->abort = 1;
                report_failure(sb, W4A8_ERR_TIMEOUT, where);
                return false;
            }
        }
    }
}
// All lanes of a warp wait and agree on the outcome.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, Control *ctl, StatusBlock *sb, int where, int pause = 0)
{
    return __all_sync(0xffffffffu, try_wait(bar, parity) || wait_long(bar, parity, ctl, sb, where, pause));
}

// The share of the work list a CTA walks through: the list is, for every sequence, row tile and key
// head in this order, kLead places and then the units that the tile's rows see (at least one place).
template <int FORM>
struct Walk {
    static constexpr bool WIDE = FORM != kPlain;
    using View = View<FORM>;
    const KvAttnArgs &a;
    const Schedule &sc;
    const bool by_items;                       // the list is that of whole items, a place each
    long long at, end, off;                    // place on the list, end of the share, place inside (sequence, tile)
    int b, tile;
    Seq s;
    bool loaded;
    // the current piece
    int h, rows, i_first, lo, first, few, units, from, count;     // few: units of sinks, among `units`
    long long first_unit;                      // the item's first unit on the list
    bool whole;

    __device__ Walk(const KvAttnArgs &a_, const Schedule &sc_, bool by_items_) : a(a_), sc(sc_), by_items(FORM == kSinks && by_items_), loaded(false) {}

    __device__ static int tiles_of(const Seq &s, int group) { return (int)(((long long)s.n * group + kRows - 1) / kRows); }
    __device__ static void span(const KvAttnArgs &a, const Schedule &sc, const Seq &s, int tile, int &i_first, int &i_last, int &rows,
                                int &lo, int &first, int &few, int &units)
    {
        rows = (int)min((long long)kRows, (long long)s.n * sc.group.d - (long long)tile * kRows);
        i_first = sc.group.div(tile * kRows);
        i_last = sc.group.div(tile * kRows + rows - 1);
        const View sight(a, s);
        few = 0;
        if constexpr (WIDE) {
            lo = sight.tile_lo(i_first);
            first = lo >> kUnitShift;
            const int hi = sight.tile_hi(i_last);
            few = sink_units(min(sight.sinks, hi), first, kUnitShift);
            units = few + max(0, ((hi + kUnit - 1) >> kUnitShift) - first);
        } else {
            lo = sight.lo(i_first);
            first = lo >> kUnitShift;
            units = max(0, ((sight.hi(i_last) + kUnit - 1) >> kUnitShift) - first);
        }
    }
    // Places of an item of row tile t of a sequence (0 behind the last tile), of all items of it.
    __device__ static int item_places(const KvAttnArgs &a, const Schedule &sc, const Seq &s, int t)
    {
        if (t >= tiles_of(s, (int)sc.group.d)) return 0;
        int i0, i1, rows, lo, first, few, units;
        span(a, sc, s, t, i0, i1, rows, lo, first, few, units);
        return kLead + max(units, 1);
    }
    __device__ static long long tile_places(const KvAttnArgs &a, const Schedule &sc, const Seq &s, int t, bool by_items = false)
    {
        const int places = item_places(a, sc, s, t);
        return (long long)a.cache.heads * (by_items ? min(places, 1) : places);
    }
    __device__ void start(int b0, int tile0, long long off0, long long begin, long long end_)
    {
        b = b0;
        tile = tile0;
        off = off0;
        at = begin;
        end = end_;
        if (at < end) {
            s = load_seq(a, b, sc.sb);
            loaded = true;
        }
    }
    // Moves to the next piece with at least one unit (or the one place of an item without units).
    __device__ bool next()
    {
        while (at < end) {
            if (!loaded) {
                s = load_seq(a, b, sc.sb);
                loaded = true;
                tile = 0;
            }
            if (tile >= tiles_of(s, (int)sc.group.d)) {
                ++b;
                loaded = false;
                continue;
            }
            int i_last;
            span(a, sc, s, tile, i_first, i_last, rows, lo, first, few, units);
            const int body = max(units, 1), length = by_items ? 1 : kLead + body;
            if (off >= (long long)a.cache.heads * length) {
                off -= (long long)a.cache.heads * length;
                ++tile;
                continue;
            }
            h = (int)quotient(off, length);
            const int in = (int)(off - (long long)h * length);
            const int here = (int)min((long long)(length - in), end - at);
            from = max(in - kLead, 0);
            count = by_items ? body : max(in + here - kLead, 0) - from;
            first_unit = at - in + kLead;
            at += here;
            off += here;
            if (count <= 0) continue;
            whole = count == body;
            count = min(count, units - from);  // an item without units has nothing to walk
            return true;
        }
        return false;
    }
};

// e such that x 2^-e is in [2^14, 2^15), the top of binary16's range; both powers normal in binary32.
__device__ __forceinline__ int query_exponent(float x) { return min(max((int)((__float_as_uint(x) >> 23) & 255u) - 127 - 14, -100), 113); }

__device__ __forceinline__ float power_of_two(int e)
{
    return __uint_as_float(e >= -126 ? (uint32_t)(127 + e) << 23 : e >= -149 ? 1u << (149 + e) : 0u);
}

// Eight elements of the output in their order, from element `at` of O on.
__device__ __forceinline__ void store_eight(const KvAttnArgs &a, size_t at, const float (&x)[8])
{
    uint4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float top = a.o_bf16 ? __uint_as_float(0x7f7f0000u) : 65504.0f;
        const float y0 = fminf(fmaxf(x[2 * k], -top), top), y1 = fminf(fmaxf(x[2 * k + 1], -top), top);
        if (a.o_bf16) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(y0, y1);
            (&o.x)[k] = *reinterpret_cast<const uint32_t *>(&z);
        } else (&o.x)[k] = pack_half2(y0, y1);
    }
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.O) + at) = o;
}

template <int D, int FORM>
__global__ void __launch_bounds__(kThreads, 1) kv_prefill_kernel(const __grid_constant__ KvAttnArgs a, const __grid_constant__ Schedule sc)
{
    using L = Layout<D>;
    using Walk = Walk<FORM>;
    using View = View<FORM>;
    constexpr bool WIDE = FORM != kPlain;                  // sinks or a tree
    extern __shared__ uint8_t raw_smem[];
    __shared__ Control ctl_store;
    Control *ctl = &ctl_store;
    uint8_t *smem = raw_smem + ((1024u - (smem_addr(raw_smem) & 1023u)) & 1023u);
    const uint32_t base = smem_addr(smem);
    const uint32_t bars = base + L::kOffBars;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto bar = [&](int i) { return bars + 8 * i; };
    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) {
            mbar_init(bar(L::kKFull + i), kExpandWarps);
            mbar_init(bar(L::kKEmpty + i), 2);
            mbar_init(bar(L::kVFull + i), kExpandWarps);
            mbar_init(bar(L::kVEmpty + i), 2);
        }
        for (int i = 0; i < 4; ++i) {          // row tile, score buffer
            mbar_init(bar(L::kSFull + i), 1);
            mbar_init(bar(L::kPReady + i), 4);
            mbar_init(bar(L::kODone + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(L::kQFull + i), 4);
            mbar_init(bar(L::kDrain + i), 1);
        }
        mbar_init(bar(L::kQmax), kSoftmaxWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(L::kPieceFull + i), 1);
            mbar_init(bar(L::kPieceEmpty + i), kSoftmaxWarps + kExpandWarps + 2);
        }
        ctl->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&ctl->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    allow_dependents();
    dependent_wait();

    // ---- this CTA's share of the list: a warp takes a run of sequences, its lanes their row tiles ----
    const int batch = a.batch.batch;
    const int chunk = (batch + kWarps - 1) / kWarps;
    const int b_first = min(batch, warp * chunk), b_last = min(batch, b_first + chunk);
    long long mine = 0;
    int my_items = 0, longest = 0;
    for (int b = b_first; b < b_last; ++b) {
        const Seq s = load_seq(a, b, sc.sb);
        if (FORM == kTree && s.n > 32 * a.tree_words) report_failure(sc.sb, W4A8_ERR_BAD_TABLE, b);
        const int tiles = Walk::tiles_of(s, (int)sc.group.d);
        for (int t = 0; t < tiles; t += 32) {
            const int places = Walk::item_places(a, sc, s, t + lane);
            mine += (long long)a.cache.heads * places;
            if (FORM == kSinks) longest = max(longest, places);
        }
        if (FORM == kSinks) my_items = min(my_items + (int)min((long long)tiles * a.cache.heads, 1ll << 20), 1 << 20);     // (as many as matter)
    }
    if (FORM == kSinks) {
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 0) {
            ctl->warp_items[warp] = my_items;
            ctl->warp_longest[warp] = longest;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) ctl->warp_len[warp] = mine;
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = ctl->tmem;
    long long total = 0, before = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += ctl->warp_len[w];
        total += ctl->warp_len[w];
    }
    long long per = max(quotient(total + gridDim.x - 1, gridDim.x), 4ll);
    bool by_items = false;
    if (FORM == kSinks) {
        // Where items are alike (every row tile lies beyond its window) and about as many as CTAs, a CTA takes one item: nothing is joined.
        int n_items = 0, items_before = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) items_before += ctl->warp_items[w];
            n_items += ctl->warp_items[w];
            longest = max(longest, ctl->warp_longest[w]);
        }
        if (n_items <= (int)gridDim.x && longest <= per + (2 * n_items > (int)gridDim.x ? kTwoParts : kOnePart)) {
            by_items = true;
            per = 1;
            total = n_items;
            before = items_before;
            mine = my_items;
        }
    }
    const long long begin = (long long)blockIdx.x * per, end = min(total, begin + per);
    if (begin < total && begin >= before && begin < before + mine) {
        long long at = before;
        bool found = false;
        for (int b = b_first; b < b_last && !found; ++b) {
            const Seq s = load_seq(a, b, sc.sb);
            const int tiles = Walk::tiles_of(s, (int)sc.group.d);
            for (int t = 0; t < tiles && !found; t += 32) {
                const long long n = Walk::tile_places(a, sc, s, t + lane, by_items);
                long long upto = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                if (begin >= at + upto - n && begin < at + upto) {
                    ctl->found_b = b;
                    ctl->found_tile = t + lane;
                    ctl->found_off = begin - (at + upto - n);
                }
                at += __shfl_sync(0xffffffffu, upto, 31);
                found = begin < at;
            }
        }
    }
    __syncthreads();
    const uint32_t tmem_s = tmem, tmem_o = tmem + 256;

    // 96 registers per thread at launch, split anew among the five warpgroups: 2 x 136 + 2 x 72 + 64 = 5 x 96
    if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        // ------------------------------------------------------------------ softmax: a thread per row
        const int w = warp >> 2, r = tid;                  // row tile, row of the 256
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;      // this warp's 32 lanes of tensor memory
        const uint32_t s_base = tmem_s + w * 128 + quarter, o_addr = tmem_o + w * D + quarter;
        const uint32_t q_tile = base + w * L::kQTile;
        uint32_t unit_no = 0, item_no = 0;
        bool ok = true;
        // The output product of unit number n.  Its barrier (one per parity of n) knows one phase: the product of
        // n - 2 went to the tensor cores before the scores of n and is complete when these are here, and that of n + 2
        // cannot start before this warp has delivered later weights.
        auto wait_output = [&](uint32_t n) {
            return wait_warp(bar(L::kODone + 2 * w + (n & 1)), (n >> 1) & 1, ctl, sc.sb, kWaitSite + 3);
        };
        for (uint32_t piece_no = 0;; ++piece_no) {
            if (!(ok = wait_warp(bar(L::kPieceFull + (piece_no & 1)), (piece_no >> 1) & 1, ctl, sc.sb, kWaitSite + 12))) break;
            const volatile Piece &pc = ctl->piece[piece_no & 1];
            const int count = pc.count;
            if (count < 0) break;
            const Seq s = {pc.row0, pc.n, pc.len};
            const View sight(a, s);
            const int few = pc.few;
            const int flat = pc.tile * kRows + r, i = sc.group.div(flat);
            const int head = pc.h * (int)sc.group.d + flat - i * (int)sc.group.d;
            const bool in = r < pc.rows;
            int row_hi, row_lo;
            if constexpr (WIDE) row_hi = in ? sight.row_hi(i) : 0, row_lo = in ? sight.row_lo(i) : 0;
            else row_hi = in ? sight.hi(i) : s.len, row_lo = in ? sight.lo(i) : 0;
            float m = kNoReference, l = 0.0f;
            if (count > 0) {
                // ---- queries to the operand tile, scaled by a power of two to the top of binary16's range ----
                // (the lanes of a row group take the 16-byte pieces of a row, so that a load touches whole lines)
                constexpr int kPer = D / 8, kTogether = 32 / kPer;   // lanes per row, rows at a time
                const int c = lane % kPer;
                uint4 raw[kPer];
                uint32_t row_max[kPer];                    // magnitudes, as their 15 bits
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int at = (r & ~31) + k * kTogether + lane / kPer, q_flat = pc.tile * kRows + at, q_i = sc.group.div(q_flat);
                    const int q_head = pc.h * (int)sc.group.d + q_flat - q_i * (int)sc.group.d;
                    raw[k] = make_uint4(0u, 0u, 0u, 0u);
                    if (at < pc.rows)
                        raw[k] = __ldca(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.Q) + (size_t)(s.row0 + q_i) * a.q_stride +
                                                                       (size_t)q_head * D) + c);
                }
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    uint32_t v = 0u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v = __vmaxu2(v, (&raw[k].x)[e] & 0x7fff7fffu);
                    row_max[k] = max(v & 0xffffu, v >> 16);
                }
                // the lanes of a row group reduce their rows together: lane c is left with the maximum of its c-th
#pragma unroll
                for (int o = kPer / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int k = 0; k < o; ++k) {
                        const uint32_t send = (lane & o) ? row_max[k] : row_max[k + o], keep = (lane & o) ? row_max[k + o] : row_max[k];
                        row_max[k] = max(keep, __shfl_xor_sync(0xffffffffu, send, o));
                    }
                const float row_top = a.q_bf16 ? __uint_as_float(row_max[0] << 16) : __half2float(__ushort_as_half((unsigned short)row_max[0]));
                float amax = row_top < INFINITY ? row_top : 0.0f;
                amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
                volatile float *qmax = reinterpret_cast<float *>(smem + L::kOffQmax) + (item_no & 1) * kSoftmaxWarps;
                if (lane == 0) {
                    qmax[warp] = amax;
                    mbar_arrive(bar(L::kQmax));
                }
                if (!(ok = wait_warp(bar(L::kQmax), item_no & 1, ctl, sc.sb, kWaitSite))) break;
#pragma unroll
                for (int k = 0; k < kSoftmaxWarps; ++k) amax = fmaxf(amax, qmax[k]);
                // One power of two for the tile's 256 rows, so that a token's constants serve them all.  A row so much smaller
                // that binary16 would lose it has a power of its own; its scores are scaled back one by one.
                const int e_tile = query_exponent(amax), e_row = query_exponent(row_top);
                const bool apart = row_top > 0.0f && e_row < e_tile - kApart;
                const bool some_apart = __any_sync(0xffffffffu, apart);
                float *row_scale = reinterpret_cast<float *>(smem + L::kOffRowScale) + (r & ~31);
                row_scale[c * kTogether + lane / kPer] = apart ? power_of_two(e_row - e_tile) : 1.0f;
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int at = (r & 96) + k * kTogether + lane / kPer;     // row of the tile of 128
                    float down = power_of_two(-e_tile);
                    if (some_apart) down = power_of_two(-__shfl_sync(0xffffffffu, apart ? e_row : e_tile, (lane & ~(kPer - 1)) + k));
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t v = (&raw[k].x)[j];
                        const float2 x = a.q_bf16 ? make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u))
                                                  : __half22float2(*reinterpret_cast<const __half2 *>(&v));
                        f[2 * j] = x.x * down;
                        f[2 * j + 1] = x.y * down;
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_tile + (c >> 3) * L::kQPart + at * 128 + (((c & 7) ^ (at & 7)) << 4)),
                                 "r"(pack_half2(f[0], f[4])), "r"(pack_half2(f[1], f[5])), "r"(pack_half2(f[2], f[6])),
                                 "r"(pack_half2(f[3], f[7]))
                                 : "memory");
                }
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::kQFull + w));
                const float scale_back = row_scale[lane];
                // rows of this warp's tile: what all of them see
                const int t_first = sc.group.div(pc.tile * kRows + w * 128);
                const int t_last = sc.group.div(pc.tile * kRows + max(w * 128, min(pc.rows, w * 128 + 128) - 1));
                int hi_min, lo_max;
                if constexpr (WIDE) hi_min = sight.all_hi(t_first), lo_max = sight.all_lo(t_last);
                else hi_min = sight.hi(t_first), lo_max = sight.lo(t_last);
                int j0 = (WIDE && few > 0 ? pc.few0 : pc.unit0) * kUnit;
                for (int u = 0; u < count; ++u, ++unit_no, j0 += kUnit) {
                    if (WIDE && u == few && few > 0) j0 = pc.unit0 * kUnit;
                    const uint32_t slot = unit_no % kConstSlots;
                    // (the scores were issued behind the unit's keys, and those behind its constants)
                    if (!(ok = wait_warp(bar(L::kSFull + 2 * w + (unit_no & 1)), (unit_no >> 1) & 1, ctl, sc.sb, kWaitSite + 2))) break;
                    fence_after();
                    const uint32_t ks_addr = base + L::kOffConst + slot * L::kConstBytes;
                    const uint32_t s_addr = s_base + (unit_no & 1) * kUnit;
                    const bool edge = j0 < lo_max || j0 + kUnit > hi_min;
                    // exponents of the row's weights.  (Scalar instructions: the packed binary32 ones take as long in the
                    // pipe, and the register moves that align their operands cost more than they saved.)
                    float x[kUnit];
                    tmem_load64(s_addr, x);
                    if (some_apart) {
#pragma unroll
                        for (int k = 0; k < kUnit; ++k) x[k] *= scale_back;
                    }
#pragma unroll
                    for (int k = 0; k < kUnit; k += 4) {
                        const float4 f = load_shared4(ks_addr + 4 * k), g = load_shared4(ks_addr + 4 * (kUnit + k));
                        x[k] = fmaf(x[k], f.x, g.x);
                        x[k + 1] = fmaf(x[k + 1], f.y, g.y);
                        x[k + 2] = fmaf(x[k + 2], f.z, g.z);
                        x[k + 3] = fmaf(x[k + 3], f.w, g.w);
                    }
                    if (WIDE && edge) {
                        if constexpr (WIDE) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint32_t seen = in ? sight.visible(i, row_lo, row_hi, j0 + 32 * half) : 0u;
#pragma unroll
                                for (int k = 0; k < 32; ++k) x[32 * half + k] = seen >> k & 1u ? x[32 * half + k] : -INFINITY;
                            }
                        }
                    } else if (edge) {
                        const int lo_off = j0 - row_lo;
                        const uint32_t span = (uint32_t)max(row_hi - row_lo, 0);
#pragma unroll
                        for (int k = 0; k < kUnit; ++k) x[k] = (uint32_t)(lo_off + k) < span ? x[k] : -INFINITY;
                    }
                    float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
                    for (int k = 0; k < kUnit; k += 4) {
                        top0 = max3(top0, x[k], x[k + 1]);
                        top1 = max3(top1, x[k + 2], x[k + 3]);
                    }
                    const float top = fmaxf(top0, top1);
                    const bool fresh = m == kNoReference;
                    const bool full = l > kFull, over = full || top > (fresh ? kNoReference : m + kSlack);
                    if (__any_sync(0xffffffffu, over)) {     // move the reference and scale what has been summed
                        const float to = over ? fmaxf(top - kRoom, full ? m + kShift : kNoReference) : m;
                        const float keep = fresh ? 0.0f : ex2(m - to);
                        m = to;
                        l *= keep;
                        if (u > 0) {
                            if (!(ok = wait_output(unit_no - 1))) break;
                            fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                uint32_t v[32];
                                tmem_load32(o_addr + 32 * c, v);
#pragma unroll
                                for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * keep);
                                tmem_store32(o_addr + 32 * c, v);
                            }
                        }
                    }
                    const float ref = m == kNoReference ? 0.0f : m;
                    uint32_t pk[kUnit / 2];
                    float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
                    for (int k = 0; k < kUnit; k += 4) {
                        const float4 g = load_shared4(ks_addr + 4 * (2 * kUnit + k));
                        const float x0 = ex2(x[k] - ref), x1 = ex2(x[k + 1] - ref), x2 = ex2(x[k + 2] - ref), x3 = ex2(x[k + 3] - ref);
                        sum0 = fmaf(x0, g.x, sum0);
                        sum1 = fmaf(x1, g.y, sum1);
                        sum0 = fmaf(x2, g.z, sum0);
                        sum1 = fmaf(x3, g.w, sum1);
                        pk[k / 2] = pack_half2(x0, x1);
                        pk[k / 2 + 1] = pack_half2(x2, x3);
                    }
                    l += sum0 + sum1;
                    tmem_store32(s_addr, pk);
                    tmem_store_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::kPReady + 2 * w + (unit_no & 1)));
                }
                if (!ok) break;
                if (!(ok = (count < 2 || wait_output(unit_no - 2)) && wait_output(unit_no - 1))) break;
                fence_after();
                ++item_no;
            }
            // ---- this row's output: -2 O / l, or a part of it ----
            const bool mine_only = pc.whole;
            float *part = sc.partials + ((size_t)blockIdx.x * 2 + pc.slot) * (kRows * (D + 2));
            const float inv = l > 0.0f ? __fdiv_rn(-2.0f, l) : 0.0f;
            const size_t out_at = ((size_t)(s.row0 + i) * a.q_heads + head) * D;
            // place of this thread's first four columns in a part, in quads: [warp][quad of columns][lane]
            const int quads_at = warp * (D / 4) * 32 + lane;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t v[32];
                if (count > 0) tmem_load32(o_addr + 32 * c, v);
                else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = 0u;
                }
                if (!mine_only) {
                    if (in)
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        __stcg(reinterpret_cast<uint4 *>(part + 2 * kRows) + quads_at + (8 * c + k / 4) * 32, make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]));
                } else if (in) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {        // columns hold the elements 0, 4, 1, 5, 2, 6, 3, 7 of eight
                        const float x[8] = {__uint_as_float(v[k]) * inv, __uint_as_float(v[k + 2]) * inv, __uint_as_float(v[k + 4]) * inv,
                                            __uint_as_float(v[k + 6]) * inv, __uint_as_float(v[k + 1]) * inv, __uint_as_float(v[k + 3]) * inv,
                                            __uint_as_float(v[k + 5]) * inv, __uint_as_float(v[k + 7]) * inv};
                        store_eight(a, out_at + 32 * c + k, x);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(L::kPieceEmpty + (piece_no & 1)));
            if (!in) continue;
            if (mine_only) {
                if (a.lse) a.lse[out_at / D] = l > 0.0f ? (m + lg2(l)) * kLn2 : -INFINITY;
            } else {
                __stcg(part + r, m);
                __stcg(part + kRows + r, l);
            }
        }
    } else if (warp < kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ------------------------------------------------------------------ expansion of the codes
        const int id = tid - 32 * kSoftmaxWarps, tk = id & (kUnit - 1), quarter = id >> kUnitShift;
        constexpr int KW = D / 32;                         // words of a quarter of a token's key codes
        constexpr int CB = D / 16;                         // bytes of a value slice
        ExpandConsts ek = {kNibble, kMinusEight};
        asm volatile("" : "+r"(ek.nibble), "+r"(ek.minus_eight));
        // where this thread's operand pieces go in a tile of keys or values
        uint32_t place[KW];
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            const int c = quarter * KW + k;
            place[k] = base + L::kOffK + (c >> 3) * L::kPartBytes + tk * 128 + (((c & 7) ^ (tk & 7)) << 4);
        }
        const int page_bits = a.cache.page_shift - 4, in_page = (1 << page_bits) - 1;
        const size_t page_bytes = a.cache.page_bytes();
        uint32_t unit_no = 0, item_no = 0;
        bool ok = true;
        for (uint32_t piece_no = 0;; ++piece_no) {
            if (!(ok = wait_warp(bar(L::kPieceFull + (piece_no & 1)), (piece_no >> 1) & 1, ctl, sc.sb, kWaitSite + 13))) break;
            const volatile Piece &pc = ctl->piece[piece_no & 1];
            const int count = pc.count, unit0 = pc.unit0, lo = pc.lo, len = pc.len, seq = pc.b;
            const uint8_t *head_base = a.cache.pages + ((size_t)pc.h << a.cache.page_shift) * (D + 8);
            __syncwarp();
            if (count >= 0 && lane == 0) mbar_arrive(bar(L::kPieceEmpty + (piece_no & 1)));
            if (count < 0) break;
            if (count == 0) continue;
            const int last_block = (len - 1) >> 4;
            const int32_t *table = a.batch.page_table + (size_t)seq * a.batch.max_pages;
            // Block of this thread's token of unit u of the piece; behind the end the last one.  In front of what the tile
            // sees, in the first unit only, the first one that it sees: the page of the other may be gone.
            // (Extended: in front of the window as behind the sinks.)
            int near = 0;
            if constexpr (WIDE) near = View(a, {pc.row0, pc.n, len}).sinks;
            const int sink_block = near > 0 ? (near - 1) >> 4 : -1;
            const int few = pc.few, few0 = pc.few0;
            auto unit_at = [&](int u) { return !WIDE ? unit0 + u : u < few ? few0 + u : unit0 + u - few; };
            auto block_no = [&](int u) {
                int blk = min(unit_at(u) * (kUnit / 16) + (tk >> 4), last_block);
                if (WIDE && blk > sink_block) blk = max(blk, lo >> 4);
                return blk;
            };
            auto page_of = [&](int blk) {
                int page = __ldca(table + (blk >> page_bits));
                if ((unsigned)page >= (unsigned)a.cache.num_pages) {
                    report_failure(sc.sb, W4A8_ERR_BAD_TABLE, seq);
                    page = 0;
                }
                return page;
            };
            uint32_t kc[KW];
            uint32_t vc[2][CB / 4], kw = 0, vw = 0;
            auto block_of = [&](int blk, int page) {
                return head_base + (size_t)page * page_bytes + (size_t)(blk & in_page) * (16 * (D + 8));
            };
            const int t = tk & 15;
            auto fetch_keys = [&](const uint8_t *p) {
                const uint8_t *q = p + t * (D / 2) + quarter * (D / 8);
                if constexpr (KW == 4) {
                    const uint4 x = __ldca(reinterpret_cast<const uint4 *>(q));
                    kc[0] = x.x; kc[1] = x.y; kc[2] = x.z; kc[3] = x.w;
                } else {
                    const uint2 x = __ldca(reinterpret_cast<const uint2 *>(q));
                    kc[0] = x.x; kc[1] = x.y;
                }
                kw = __ldca(reinterpret_cast<const uint32_t *>(p + 16 * D + 4 * t));
                vw = __ldca(reinterpret_cast<const uint32_t *>(p + 16 * D + 64 + 4 * t));
            };
            auto fetch_values = [&](const uint8_t *p) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint8_t *q = p + 8 * D + (((t >> 3) * 8 + quarter * 2 + k) * 8 + (t & 7)) * CB;
                    if constexpr (CB == 8) {
                        const uint2 x = __ldca(reinterpret_cast<const uint2 *>(q));
                        vc[k][0] = x.x;
                        vc[k][1] = x.y;
                    } else vc[k][0] = __ldca(reinterpret_cast<const uint32_t *>(q));
                }
            };
            const int blk0 = WIDE ? block_no(0) : max(block_no(0), lo >> 4);
            const uint8_t *block = block_of(blk0, page_of(blk0));
            fetch_keys(block);
            fetch_values(block);
            int page = count > 1 ? page_of(block_no(1)) : 0;
            const int from_lo = unit0 * kUnit + tk - lo;     // place of this thread's first token behind the first that the tile sees
            const uint32_t seen = (uint32_t)(len - lo);
            if (!(ok = wait_warp(bar(L::kQmax), item_no & 1, ctl, sc.sb, kWaitSite + 4))) break;
            const volatile float *qmax = reinterpret_cast<const float *>(smem + L::kOffQmax) + (item_no & 1) * kSoftmaxWarps;
            float amax = 0.0f;
#pragma unroll
            for (int k = 0; k < kSoftmaxWarps; ++k) amax = fmaxf(amax, qmax[k]);
            const float unit = -2.0f * (a.scale * kLog2e) * __uint_as_float((uint32_t)(127 + query_exponent(amax)) << 23);
            ++item_no;
            // Eight levels (times -1/2) of a code word; off = (16 + z) / 2 twice.
            auto levels = [&](uint32_t w, uint32_t off, uint32_t (&o)[4]) {
                const uint32_t sw = perm(w, w, 0x2301u);
                o[0] = pick_rank(w << 4, ek);
                o[1] = pick_rank(w, ek);
                o[2] = pick_rank(sw << 4, ek);
                o[3] = pick_rank(sw, ek);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t x = hadd2(o[k], off);     // -(x + 1) / 2
                    o[k] = hadd2(x, hfma2_sat(x, kMinusHalf, kQuarter));
                }
            };
            for (int u = 0; u < count; ++u, ++unit_no) {
                const uint32_t buf = unit_no % kRing, use = unit_no / kRing & 1, slot = unit_no % kConstSlots;
                bool there = (uint32_t)(from_lo + u * kUnit) < seen;             // else its words are anything
                if constexpr (WIDE) {
                    const int at = unit_at(u) * kUnit + tk;
                    there = (at >= lo || at < near) && at < len;
                }
                // ---- keys ----
                if (unit_no >= kRing && !(ok = wait_warp(bar(L::kKEmpty + buf), use ^ 1, ctl, sc.sb, kWaitSite + 5, 200))) break;
                {
                    const uint32_t off = (kw & 15u) * 0x00400040u + 0x48004800u;
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                            uint32_t o[4];
                            levels(kc[k], off, o);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place[k] + buf * L::kTile),
                                         "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3])
                                         : "memory");
                        }
                }
                if (quarter == 0) {                        // (a token behind the end or in front of the window weighs nothing)
                    float *ks = reinterpret_cast<float *>(smem + L::kOffConst + slot * L::kConstBytes) + tk;
                    const float step = __uint_as_float(vw & ~15u);
                    ks[0] = there ? __uint_as_float(kw & ~15u) * unit : 0.0f;
                    ks[kUnit] = there ? lg2(step) : -INFINITY;
                    ks[2 * kUnit] = there ? rcp(step) : 0.0f;
                }
                const uint32_t value_word = vw;
                if (u + 1 < count) {                       // the next unit's keys travel while the values are expanded
                    block = block_of(block_no(u + 1), page);
                    fetch_keys(block);
                    if (u + 2 < count) page = page_of(block_no(u + 2));
                }
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::kKFull + buf));
                // ---- values ----
                if (unit_no >= kRing && !(ok = wait_warp(bar(L::kVEmpty + buf), use ^ 1, ctl, sc.sb, kWaitSite + 6, 200))) break;
                {
                    const uint32_t off = (value_word & 15u) * 0x00400040u + 0x48004800u;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int j = 0; j < CB / 4; ++j) {
                            uint32_t o[4];
                            levels(vc[k][j], off, o);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place[k * (CB / 4) + j] + (kRing + buf) * L::kTile),
                                         "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3])
                                         : "memory");
                        }
                }
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::kVFull + buf));
                if (u + 1 < count) fetch_values(block);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ------------------------------------------------------------------ MMA issue
        if (warp < kListWarp && lane == 0) {
            const int w = warp - kMmaWarp;                 // row tile
            constexpr uint32_t idesc_s = instr_desc(kUnit, 0), idesc_o = instr_desc(D, 1);
            uint32_t unit_no = 0, item_no = 0;
            bool ok = true;
            auto wait = [&](int i, uint32_t parity, int where) {
                return try_wait(bar(i), parity) || wait_long(bar(i), parity, ctl, sc.sb, kWaitSite + where, 0);
            };
            const uint32_t q_tile = desc_low(base + w * L::kQTile, 16), s_tile = tmem_s + w * 128, o_tile = tmem_o + w * D;
            auto scores = [&](uint32_t n) {                // S of unit number n
                const uint32_t d = s_tile + (n & 1) * kUnit;
                uint32_t q = q_tile, k = desc_low(base + L::kOffK + n % kRing * L::kTile, 16);
#pragma unroll 1
                for (int part = 0; part < L::kHalves; ++part, q += L::kQPart >> 4, k += L::kPartBytes >> 4) {
#pragma unroll
                    for (uint32_t x = 0; x < 4; ++x) mma_ss(d, q + 2 * x, k + 2 * x, idesc_s, part + x);
                }
                commit(bar(L::kSFull + 2 * w + (n & 1)));
                commit(bar(L::kKEmpty + n % kRing));
            };
            auto output = [&](uint32_t n, uint32_t accumulate) {
                const uint32_t v = desc_low(base + L::kOffV + n % kRing * L::kTile, L::kPartBytes), p = s_tile + (n & 1) * kUnit;
#pragma unroll
                for (uint32_t x = 0; x < kUnit / 16; ++x) mma_ts(o_tile, p + 8 * x, v + x * (2048 >> 4), idesc_o, accumulate + x);
                commit(bar(L::kODone + 2 * w + (n & 1)));
                commit(bar(L::kVEmpty + n % kRing));
            };
            for (uint32_t piece_no = 0;; ++piece_no) {
                if (!(ok = wait(L::kPieceFull + (piece_no & 1), (piece_no >> 1) & 1, 14))) break;
                const int n = reinterpret_cast<const volatile Piece &>(ctl->piece[piece_no & 1]).count;
                if (n < 0) break;
                mbar_arrive(bar(L::kPieceEmpty + (piece_no & 1)));
                if (n == 0) continue;
                if (!(ok = wait(L::kQFull + w, item_no & 1, 7) && wait(L::kKFull + unit_no % kRing, unit_no / kRing & 1, 8))) break;
                fence_after();
                scores(unit_no);
                // the scores of a unit are computed while the softmax of the one before runs
                for (int u = 0; u < n; ++u, ++unit_no) {
                    const uint32_t next = unit_no + 1;
                    if (u + 1 < n) {
                        if (!(ok = wait(L::kKFull + next % kRing, next / kRing & 1, 8))) break;
                        fence_after();
                        scores(next);
                    }
                    if (!(ok = wait(L::kVFull + unit_no % kRing, unit_no / kRing & 1, 9) &&
                               wait(L::kPReady + 2 * w + (unit_no & 1), (unit_no >> 1) & 1, 10)))
                        break;
                    fence_after();
                    output(unit_no, u);
                }
                ++item_no;
            }
            if (!ok) {                                     // nothing of this CTA may still run when it gives its memory back
                commit(bar(L::kDrain + w));
                unsigned long long t0, t;
                asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
                do {
                    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
                } while (!try_wait(bar(L::kDrain + w), 0) && t - t0 < kWaitNs / 10);
            }
        }
        if (warp == kListWarp && lane == 0) {
            // -------------------------------------------------------------- the pieces of this CTA's share
            Walk walk(a, sc, by_items);
            walk.start(ctl->found_b, ctl->found_tile, ctl->found_off, begin, max(begin, end));
            Shared shared = {};
            for (uint32_t piece_no = 0;; ++piece_no) {
                const bool more = walk.next();
                if (piece_no >= 2 && !try_wait(bar(L::kPieceEmpty + (piece_no & 1)), (piece_no >> 1 & 1) ^ 1) &&
                    !wait_long(bar(L::kPieceEmpty + (piece_no & 1)), (piece_no >> 1 & 1) ^ 1, ctl, sc.sb, kWaitSite + 15, 1000))
                    break;
                Piece p = {};
                p.count = -1;
                if (more) {
                    const int body = max(walk.units, 1);
                    p.b = walk.b;
                    p.h = walk.h;
                    p.tile = walk.tile;
                    p.rows = walk.rows;
                    p.row0 = walk.s.row0;
                    p.n = walk.s.n;
                    p.len = walk.s.len;
                    p.unit0 = walk.first + (WIDE ? max(walk.from - walk.few, 0) : walk.from);
                    p.count = walk.count;
                    p.lo = walk.lo;
                    if constexpr (WIDE) {
                        p.few0 = walk.from;
                        p.few = max(min(walk.few - walk.from, walk.count), 0);
                    }
                    p.whole = walk.whole;
                    p.slot = walk.first_unit <= begin ? 0 : 1;
                    if (!walk.whole && walk.first_unit >= begin) {       // begins here and ends in a later share
                        shared.parts = (int)(quotient(walk.first_unit + body - 1, per) - (long long)blockIdx.x) + 1;
                        shared.inside = walk.first_unit > begin;
                        shared.row0 = walk.s.row0;
                        shared.h = walk.h;
                        shared.tile = walk.tile;
                        shared.rows = walk.rows;
                    }
                }
                ctl->piece[piece_no & 1] = p;
                mbar_arrive(bar(L::kPieceFull + (piece_no & 1)));
                if (!more) break;
            }
            sc.shared[blockIdx.x] = shared;
        }
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// Joins the parts of the items that several CTAs shared, in list order.  A kernel of its own spreads this over
// the GPU: left to the CTA that finishes an item last, the parts (131 KB each) pass through one SM, some 1.2 us
// per part.  Block (x, y): rows 32 x .. 32 x + 31 of the item that begins in share y; a warp takes 16 columns.
constexpr int kJoinColumns = 16;
template <int D>
__global__ void __launch_bounds__(2 * D) kv_prefill_join_kernel(const __grid_constant__ KvAttnArgs a, const __grid_constant__ Schedule sc)
{
    allow_dependents();
    dependent_wait();
    const Shared item = sc.shared[blockIdx.y];
    const int lane = threadIdx.x & 31, c = threadIdx.x / 32 * kJoinColumns, r = blockIdx.x * 32 + lane;
    if (item.parts == 0 || r >= item.rows) return;
    constexpr size_t kPart = kRows * (D + 2);
    constexpr int kQuads = kJoinColumns / 4;
    const float *rest = sc.partials + (size_t)blockIdx.y * 2 * kPart, *first = rest + (item.inside ? kPart : 0);
    auto part = [&](int k) { return k == 0 ? first : rest + (size_t)k * 2 * kPart; };
    struct Slice {
        float m, l;
        float4 y[kQuads];
    };
    auto load = [&](int k, Slice &x) {
        const float *from = part(k);
        x.m = __ldcg(from + r);
        x.l = __ldcg(from + kRows + r);
        const float4 *at = reinterpret_cast<const float4 *>(from + 2 * kRows) + (blockIdx.x * (D / 4) + c / 4) * 32 + lane;
#pragma unroll
        for (int q = 0; q < kQuads; ++q) x.y[q] = __ldcg(at + q * 32);
    };
    // (an item has two parts as a rule: both are loaded before anything is computed)
    Slice x0, x1;
    load(0, x0);
    if (item.parts > 1) load(1, x1);
    else x1.m = kNoReference, x1.l = 0.0f;
    float top = fmaxf(x0.m, x1.m), most = fmaxf(fmaxf(x0.l, x1.l), 0.0f);
#pragma unroll 4
    for (int k = 2; k < item.parts; ++k) {
        top = fmaxf(top, __ldcg(part(k) + r));
        most = fmaxf(most, __ldcg(part(k) + kRows + r));
    }
    if (most > kFull) top += kLift;            // the sums below fit whatever the parts hold
    float acc[kJoinColumns], lsum = 0.0f;
#pragma unroll
    for (int k = 0; k < kJoinColumns; ++k) acc[k] = 0.0f;
    auto add = [&](const Slice &x) {
        const float f = ex2(x.m - top);
        lsum = fmaf(x.l, f, lsum);
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            acc[4 * q] = fmaf(x.y[q].x, f, acc[4 * q]);
            acc[4 * q + 1] = fmaf(x.y[q].y, f, acc[4 * q + 1]);
            acc[4 * q + 2] = fmaf(x.y[q].z, f, acc[4 * q + 2]);
            acc[4 * q + 3] = fmaf(x.y[q].w, f, acc[4 * q + 3]);
        }
    };
    add(x0);
    if (item.parts > 1) add(x1);
#pragma unroll 2
    for (int k = 2; k < item.parts; ++k) {
        load(k, x0);
        add(x0);
    }
    const float inv = lsum > 0.0f ? __fdiv_rn(-2.0f, lsum) : 0.0f;
    const int flat = item.tile * kRows + r, i = sc.group.div(flat);
    const size_t row = (size_t)(item.row0 + i) * a.q_heads + item.h * (int)sc.group.d + flat - i * (int)sc.group.d;
#pragma unroll
    for (int k = 0; k < kJoinColumns; k += 8) {
        const float y[8] = {acc[k] * inv, acc[k + 2] * inv, acc[k + 4] * inv, acc[k + 6] * inv,
                            acc[k + 1] * inv, acc[k + 3] * inv, acc[k + 5] * inv, acc[k + 7] * inv};
        store_eight(a, row * D + c + k, y);
    }
    if (a.lse && c == 0) a.lse[row] = lsum > 0.0f ? (top + lg2(lsum)) * kLn2 : -INFINITY;
}

template <int D, int FORM>
cudaError_t launch_form(const KvAttnArgs &a, const Schedule &sc, int ctas, cudaStream_t st)
{
    static std::atomic<int> raised[kMaxDevices];
    cudaError_t e = raise_smem_limit(kv_prefill_kernel<D, FORM>, Layout<D>::kSmem, raised);
    if (e == cudaSuccess) e = launch_overlapped(kv_prefill_kernel<D, FORM>, dim3(ctas), dim3(kThreads), Layout<D>::kSmem, st, a, sc);
    if (e == cudaSuccess) e = launch_overlapped(kv_prefill_join_kernel<D>, dim3(kRows / 32, ctas), dim3(2 * D), 0, st, a, sc);
    return e;
}
template <int D>
cudaError_t launch(const KvAttnArgs &a, const Schedule &sc, int ctas, cudaStream_t st)
{
    switch (form_of(a)) {
    case kTree: return launch_form<D, kTree>(a, sc, ctas, st);
    case kSinks: return launch_form<D, kSinks>(a, sc, ctas, st);
    default: return launch_form<D, kPlain>(a, sc, ctas, st);
    }
}

}  // namespace

// Status block, two parts per CTA, the shared items.  (The counters of the decode form are left alone.)
size_t kv_prefill_workspace(int D)
{
    const int sms = device_sms();
    return sizeof(StatusBlock) + kv_counters_bytes(sms) + (size_t)sms * (2 * kRows * (D + 2) * sizeof(float) + sizeof(Shared));
}

cudaError_t launch_kv_prefill(const KvAttnArgs &a, uint8_t *workspace, cudaStream_t st)
{
    const int sms = device_sms();
    float *partials = reinterpret_cast<float *>(workspace + sizeof(StatusBlock) + kv_counters_bytes(sms));
    const Schedule sc = {reinterpret_cast<StatusBlock *>(workspace), partials,
                         reinterpret_cast<Shared *>(partials + (size_t)sms * 2 * kRows * (a.cache.D + 2)),
                         Divisor((uint32_t)(a.q_heads / a.cache.heads))};
    return a.cache.D == 64 ? launch<64>(a, sc, sms, st) : launch<128>(a, sc, sms, st);
}

}  // namespace w4a8
