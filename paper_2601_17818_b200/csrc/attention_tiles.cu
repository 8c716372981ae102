// Attention over K and V in bf16 for many query rows (prompts, questions, large trees): tcgen05, two tiles of 128 query rows a CTA.
//
// A tile's rows are as many tokens as 128 / R query heads of a stored one allow (row t R + r), brought by one tensor copy; the two tiles of an item
// read the same blocks of 128 tokens.  Blocks end where the last row's window (or the sinks) ends, so that nothing behind a sequence is read;
// what a first block reaches back beyond its segment, or the sequence, is masked.  Of a block that a tile sees in part only the 32-token
// columns that it sees are worked on.
//   warps 0-3, 4-7  softmax of a tile, a thread a row: logits from tensor memory, weights back to where the logits were, as the operand of
//                   the second product.  Weights are made by the maximum so far, set high above the logits, while the block's own is looked for; only when a
//                   logit comes near it is it moved, the sums so far with it, and the weights are made anew
//   warp 8          tensor copies: queries, then K and V of a block in turn through a ring.  Rows of V that are no numbers must not reach rows that do
//                   not see them, and 0 times NaN does: blocks that are masked are looked through, such rows taken out and added again at the end
//                   for those who see them
//   warp 9          products: PV(A), QK(A), PV(B), QK(B): while one tile's softmax runs, the other's products do
// A CTA takes items in turn, the next item's first products under the last one's output.  Where items are fewer than SMs, a cluster of up to eight CTAs
// shares an item's blocks and joins its parts in shared memory.
// Bound by the chain of a tile, logits to weights to products, which one other tile does not fill, and tensor memory holds no third: some 3300 cycles for a
// block of two tiles, of which the tensor cores work 2048 and the units of exponentials as many.  16512 tokens x 28 heads of 128, window 4096: 870-930 us
// (0.93-1.0 PFLOP/s, at the power limit), without a window 1902 (1.03); 2 x 4672, window 1024: 183; 8 x up to 704 x 32 heads, window 256: 71, where items' beginnings and ends count.
// Weights enter the second product in bf16, the output is divided by the sum of the unrounded ones: 0.0019-0.0023 of the output's size from 64 bits.  (By
// that of the rounded ones: 0.0018, 11 % more time.)
#include "attention.cuh"

#include <algorithm>
#include <cmath>

#include "gram.cuh"
#include "tcgen05.cuh"

namespace vitcop {
namespace {

constexpr int kTile = 128, kBlock = 128;
constexpr int kSoftmaxThreads = 256, kLoadWarp = kSoftmaxThreads / 32, kMmaWarp = kLoadWarp + 1;
// Two warps have nothing to do: registers change hands by four warps, and a row's 128 logits want more than the 168 a thread that the block is launched
// with.  (Next to 227 KB of shared memory there is no cache to spill to.)
constexpr int kThreads = kSoftmaxThreads + 128, kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(kSoftmaxThreads * kSoftmaxRegs + 128 * kOtherRegs == kThreads * 168, "registers that are asked for and not there are waited for, for ever");
constexpr int kMasked = 14;                                // blocks of an item that a tile sees in part: of either tile at most two at the end of its
                                                           // window, two where it begins, two where the sinks end; and the first
constexpr int kItemBytes = 128, kMostCtas = 8;
enum { kRoleLoad = 1, kRoleMma = 2, kRoleSoftmax = 4 };

template <int D>
struct TilesSmem {
    static constexpr int kSubs = D / 64;                               // operands are [D / 64][128 rows][128 bytes]
    static constexpr int kOperand = kSubs * 16384;
    static constexpr int kSlots = D == 128 ? 5 : 10;
    static constexpr int kQ = 0;
    static constexpr int kRing = 2 * kOperand;
    static constexpr int kBars = kRing + kSlots * kOperand;
    static constexpr int kFlags = kBars + 24 * kSlots + 144;        // behind the barriers
    static constexpr int kItems = (kFlags + 24 + 15) / 16 * 16;                        // two of them
    static constexpr int kBad = kItems + 2 * kItemBytes;        // [2][kMasked][4] words: rows of V that were taken out
    static constexpr int kBytes = kBad + 2 * kMasked * 16;
    static_assert(kBytes <= 232448);
    // parts of a cluster, where the operands were: [256 rows][D + 4], and their maxima and sums, [2][256]
    static constexpr int kPitch = D + 4;
    static constexpr int kPartEnds = 256 * kPitch * 4;
    static constexpr int kPartCounts = kPartEnds + 2 * 256 * 4;        // [256]
    static_assert(kPartCounts + 256 * 4 <= kBars);
};

struct TilesArgs {
    SeqArgs a;
    Divisor heads;                                         // heads of a sample
    int items, per_head, tokens, ctas;                     // items, and those of a head; tokens of a tile; CTAs of a cluster
    bool wide;                                             // rows of the output lie at multiples of 32 bytes
    int q_b, k_h, k_b, v_h, v_b;                           // 0 where all samples, or heads, are one, else 1
    unsigned long long wait_ns;
    int expire_roles;
    __device__ __forceinline__ unsigned long long limit_of(int role) const { return (expire_roles & role) ? 0ull : wait_ns; }
};

// As mbar_wait, for a warp.  One lane asks, the others step along: a barrier asked by 32 lanes of 16 warps holds up all else that goes through shared
// memory's pipe, and where one lane loops apart from the others the first access to tensor memory behind it takes 600 cycles.
__device__ __forceinline__ bool asked(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, 0, 0;\n\tsetp.eq.u32 q, %3, 0;\n\t"
        "@q mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(threadIdx.x & 31)
        : "memory");
    return __any_sync(0xffffffffu, done != 0);
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    unsigned long long t0 = 0ull;
    bool in_time = limit_ns != 0ull;
    for (uint32_t it = 1; in_time; ++it) {
        if (asked(bar, parity)) {
            __syncwarp();                                  // (a vote orders no memory: what the barrier stands for is there for the lane that asked)
            return true;
        }
        if ((it & 63u) == 0u) {                            // (reading the clock takes longer than most waits)
            const unsigned long long now = __shfl_sync(0xffffffffu, global_ns(), 0);
            if (t0 == 0ull) t0 = now;
            in_time = !__any_sync(0xffffffffu, *abort_flag != 0) && now - t0 <= limit_ns;
        }
    }
    *abort_flag = 1;
    return false;
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// One lane of a warp, the same each time.
__device__ __forceinline__ bool elected() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
// As tc_mma_bf16, the first operand in tensor memory.
__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem),
        "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Operand whose 64-element rows (128 bytes, swizzled) run along the product's N: 8 of them (steps of its K) are 1024 bytes, the next 64 of N 16384 further.
__device__ __forceinline__ uint64_t umma_desc_mn128(uint32_t smem_addr) {
    return umma_desc_k128(smem_addr) | (uint64_t)(16384u >> 4) << 16;
}
// A descriptor, its address (in 16 bytes) further on; what is not the address stays in the same register.
__device__ __forceinline__ uint64_t further(uint64_t desc, uint32_t by) {
    uint64_t d;
    asm("{\n\t.reg .b32 lo, hi;\n\tmov.b64 {lo, hi}, %1;\n\tadd.u32 lo, lo, %2;\n\tmov.b64 %0, {lo, hi};\n\t}" : "=l"(d) : "l"(desc), "r"(by));
    return d;
}
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pin32(uint32_t (&r)[32]) {   // (no use of the registers in front of the wait)
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&o)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]), "=r"(o[8]), "=r"(o[9]), "=r"(o[10]),
          "=r"(o[11]), "=r"(o[12]), "=r"(o[13]), "=r"(o[14]), "=r"(o[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The blocks of an item: first those of the sinks, then those of the window (or of the whole sequence), both counted from their end.
struct Blocks {
    Span v;
    int na, n;
    __device__ __forceinline__ int end(int k) const { return k < na ? v.a - (na - 1 - k) * kBlock : v.b1 - (n - 1 - k) * kBlock; }
    __device__ __forceinline__ int begin_of_segment(int k) const { return k < na ? 0 : v.b0; }
};
template <bool TREE>
__device__ __forceinline__ Blocks blocks_of(const SeqArgs& a, const Sample& s, int t0, int t1) {
    Blocks x;
    x.v = span_of<TREE>(a, s, t0, t1);
    x.na = (x.v.a + kBlock - 1) / kBlock;
    x.n = x.na + (x.v.b1 - x.v.b0 + kBlock - 1) / kBlock;
    return x;
}
// Columns [lo, hi) of block k that a tile works on, multiples of 32 (none: lo = hi), and whether all its rows see all of them.
struct Columns {
    int lo, hi;
    bool all;
};
__device__ __forceinline__ Columns columns_of(const Blocks& x, int k, const Span& tile) {
    const int end = x.end(k), start = end - kBlock, segment = x.begin_of_segment(k), from = max(start, segment);
    const bool front = from < tile.a, window = from < tile.b1 && end > tile.b0;
    Columns c = {0, 0, true};
    if (!front && !window) return c;
    const int lo = front ? from : max(from, tile.b0), hi = window ? min(end, tile.b1) : min(end, tile.a);
    c.lo = (lo - start) & ~31;
    c.hi = (hi - start + 31) & ~31;
    c.all = start + c.lo >= segment && tile.full(start + c.lo, start + c.hi);
    return c;
}

// Blocks first .. end - 1 of a window (a whole sequence), which all rows of a tile see all of: what most blocks are.
struct Whole {
    int first, end;
};
template <bool TREE>
__device__ __forceinline__ Whole whole_of(const Blocks& x, const Span& tile) {
    const int lo = TREE ? 0 : max(tile.all_lo, x.v.b0), hi = TREE ? tile.all_front : tile.all_hi;
    // block i ends at b1 - (n - 1 - i) 128: not behind hi, and begins not in front of lo
    const int behind = max(0, x.v.b1 - hi), room = x.v.b1 - lo - kBlock;
    Whole w = {x.n, x.n};
    if (hi > 0 && room >= 0) {
        w.end = x.n - (behind + kBlock - 1) / kBlock;
        w.first = max(x.na, x.n - 1 - room / kBlock);
    }
    return w;
}

// What a CTA works on next: two tiles of a head, as the load warp leaves it.
struct Tile {
    Span span;
    Whole whole;
    __device__ __forceinline__ Columns columns(const Blocks& x, int k) const {
        const Columns c = {0, kBlock, true};
        return k >= whole.first && k < whole.end ? c : columns_of(x, k, span);
    }
};
struct Item {
    int there, b, h, t0, len, queries, k0, k1;
    Blocks blocks;
    Tile tiles[2];
};
static_assert(sizeof(Item) == kItemBytes);

// Bits below x of a word (a shift by 32 and more leaves none).
__device__ __forceinline__ uint32_t below(int x) {
    uint32_t from;
    asm("shl.b32 %0, %1, %2;" : "=r"(from) : "r"(0xffffffffu), "r"(max(x, 0)));
    return ~from;
}
__device__ __forceinline__ uint32_t bits_of(const Seen<false>& s, int j0) { return below(s.front - j0) | (below(s.p + 1 - j0) & ~below(s.lo - j0)); }
__device__ __forceinline__ uint32_t bits_of(const Seen<true>& s, int j0) {
    const int i = j0 - s.base;                             // drafted token of bit 0
    const uint32_t drafted = i <= -32 || i >= 64 ? 0u : i < 0 ? (uint32_t)(s.bits << -i) : (uint32_t)(s.bits >> i);
    return below(s.front - j0) | (drafted & below(s.len - j0) & ~below(-j0));
}

// What tokens whose V was taken out add to a row, elements `from` .. `from` + 31: in fp32, from where they lie.
template <int D, bool TREE>
__device__ __noinline__ void add_taken_out(const SeqArgs& a, const Item& it, const Seen<TREE>& seen, const uint32_t* bad, int hq, int t, int from, float top, float (&v)[32]) {
    const __nv_bfloat16* const q = a.io.q + it.b * a.io.q_at[0] + hq * a.io.q_at[1] + t * a.io.q_at[2];
    const __nv_bfloat16* const K = a.io.K + it.b * a.io.k_at[0] + it.h * a.io.k_at[1];
    const __nv_bfloat16* const V = a.io.V + it.b * a.io.v_at[0] + it.h * a.io.v_at[1] + from;
    int n = 0;
    for (int i = it.k0; i < it.k1; ++i) {
        if (it.tiles[0].columns(it.blocks, i).all && it.tiles[1].columns(it.blocks, i).all) continue;
        const int start = it.blocks.end(i) - kBlock, segment = it.blocks.begin_of_segment(i);
        for (int w = 0; w < 4; ++w) {
            for (uint32_t left = bad[n * 4 + w]; left; left &= left - 1) {
                const int64_t j = start + w * 32 + __ffs(left) - 1;
                if (j < segment || !seen((int)j)) continue;
                float z = 0.f;
                for (int e = 0; e < D; ++e) z = fmaf(__bfloat162float(q[e]), __bfloat162float(K[j * a.io.k_at[2] + e]), z);
                const float p = ex2_approx(fmaf(a.sign ? -z : z, a.scale_log2, -top));
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = fmaf(p, __bfloat162float(V[j * a.io.v_at[2] + e]), v[e]);
            }
        }
        ++n;
    }
}

template <int D, bool TREE>
__global__ void __launch_bounds__(kThreads, 1)
attention_tiles_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ TilesArgs k) {
    using S = TilesSmem<D>;
    constexpr int kSlots = S::kSlots, kSubs = S::kSubs;
    const SeqArgs& a = k.a;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const uint32_t bar_full = base + S::kBars, bar_empty = bar_full + 8 * kSlots, bar_q = bar_empty + 8 * kSlots, bar_q_free = bar_q + 16, bar_s = bar_q_free + 8,
                   bar_p = bar_s + 16, bar_o = bar_p + 16, bar_o_free = bar_o + 16, bar_item = bar_o_free + 16, bar_done = bar_item + 16,
                   bar_drain = bar_done + 16, bar_p2 = bar_drain + 8, bar_checked = bar_p2 + 16;
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + S::kFlags);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kFlags + 4);
    volatile int* const any_bad = reinterpret_cast<volatile int*>(smem + S::kFlags + 8);           // [2 items]
    uint32_t* const bad = reinterpret_cast<uint32_t*>(smem + S::kBad);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(bar_full + 8 * i, 1);
            mbar_init(bar_empty + 8 * i, 1);
            mbar_init(bar_checked + 8 * i, 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(bar_q + 8 * x, 1);
            mbar_init(bar_s + 8 * x, 1);
            mbar_init(bar_p + 8 * x, 4);
            mbar_init(bar_p2 + 8 * x, 4);
            mbar_init(bar_o + 8 * x, 1);
            mbar_init(bar_o_free + 8 * x, 4);
            mbar_init(bar_item + 8 * x, 1);
            mbar_init(bar_done + 8 * x, kSoftmaxThreads / 32 + 1);
        }
        mbar_init(bar_q_free, 1);
        mbar_init(bar_drain, 1);
        *abort_flag = (base & 1023u) != 0;                 // (operands lie at multiples of 1024, or nothing is done)
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == kSoftmaxThreads) {
        prefetch_map(&map_q);
        prefetch_map(&map_k);
        prefetch_map(&map_v);
    }
    if (warp == kMmaWarp) tmem_alloc(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    grid_dependency_wait();
    grid_dependency_launch_dependents();
    // S(A), S(B): 128 columns each, whose first 64 take the weights; O(A), O(B): D columns each
    const auto tmem_s = [&](int x) { return tmem + x * kBlock; };
    const auto tmem_o = [&](int x) { return tmem + 2 * kBlock + x * D; };
    const int rank = blockIdx.x & (k.ctas - 1);
    uint32_t issued = 0, fetched = 0;                      // operands and items whose copies the load lane has started
    const int R = (int)a.R.d, tokens = k.tokens;
    const auto sample_in = [&](const Item& it) {
        const Sample s = {it.len, it.queries, it.len - it.queries};
        return s;
    };
    // whether there is an item n for this CTA
    const Item* const items = reinterpret_cast<const Item*>(smem + S::kItems);
    const auto item_there = [&](int n, unsigned long long lim) {
        return warp_wait(bar_item + 8 * (n & 1), (n >> 1) & 1, abort_flag, lim) && items[n & 1].there != 0;
    };

    if (warp < kLoadWarp) {
        // ------------------------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int x = warp >> 2, row = tid & (kTile - 1), tl = quotient(row, a.R), r = row - tl * R;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem_s(x) + lanes, o_at = tmem_o(x) + lanes;
        uint32_t phase_s = 0, phase_o = 0;
        const f32x2 scale2 = pack2(a.scale_log2, a.scale_log2);
        bool ok = true;
        const auto waited = [&](uint32_t bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, k.limit_of(kRoleSoftmax)); };
        const auto tell = [&](uint32_t bar) {              // what this warp has written to tensor memory is there
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        for (int n = 0; ok && item_there(n, k.limit_of(kRoleSoftmax)); ++n) {
            const Item& it = items[n & 1];
            // (made anew where it is wanted, in the blocks that are masked)
            const auto seen_by_row = [&]() {
                const int t = it.t0 + x * tokens + tl;
                return Seen<TREE>(a, sample_in(it), it.b, tl < tokens && t < it.queries ? t : it.queries);
            };
            float top = kNoLogit;                          // in powers of two: weights are 2^(logit - top), 1 at most
            f32x2 sum = pack2(0.f, 0.f);
            int count = 0;
            const Whole whole = it.tiles[x].whole;
            const int k1 = it.k1;
            for (int i = it.k0; i < k1; ++i) {
                Columns c = {0, kBlock, true};
                if (!(i >= whole.first && i < whole.end)) c = columns_of(it.blocks, i, it.tiles[x].span);
                if (c.lo == c.hi) continue;
                ok = waited(bar_s + 8 * x, phase_s);
                if (!ok) break;
                phase_s ^= 1;
                tc_fence_after();
                // Logits of rows that are not seen become -inf where they lie, 32 columns at a time and only those in which some row of the warp has
                // one: a loop, for what is unrolled over a row's registers and seldom run is fetched anew each time.
                if (!c.all || c.hi - c.lo < kBlock) {
                    const Seen<TREE> seen = seen_by_row();
                    const int start = it.blocks.end(i) - kBlock, segment = it.blocks.begin_of_segment(i);
                    uint32_t keep[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w)            // (columns that were not worked on are anything)
                        keep[w] = w * 32 >= c.lo && w * 32 < c.hi ? bits_of(seen, start + w * 32) & ~below(segment - start - w * 32) : 0u;
#pragma unroll 1
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t mine = w == 0 ? keep[0] : w == 1 ? keep[1] : w == 2 ? keep[2] : keep[3];
                        if (__all_sync(0xffffffffu, mine == 0xffffffffu)) continue;
                        uint32_t y[32];
                        tmem_ld32_issue(s_at + w * 32, y);
                        tmem_ld_wait();
                        pin32(y);
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = mine >> e & 1 ? y[e] : 0xff800000u;
                        tmem_st32(s_at + w * 32, y);
                    }
                    tmem_st_wait();
                }
                uint32_t z[4][32];
#pragma unroll
                for (int w = 0; w < 4; ++w) tmem_ld32_issue(s_at + w * 32, z[w]);
                tmem_ld_wait();
#pragma unroll
                for (int w = 0; w < 4; ++w) pin32(z[w]);
                f32x2 more = pack2(0.f, 0.f), more2 = more;
                const auto weights = [&](int w) {          // of 32 columns
                    const f32x2 top2 = pack2(-top, -top);
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float2 y = unpack2(fma2(pack2(__uint_as_float(z[w][2 * e]), __uint_as_float(z[w][2 * e + 1])), scale2, top2));
                        const float p0 = ex2_approx(y.x), p1 = ex2_approx(y.y);
                        if (e & 1) more2 = add2(more2, pack2(p0, p1));
                        else more = add2(more, pack2(p0, p1));
                        p[e] = bf16x2(p0, p1);
                    }
                    tmem_st16(s_at + w * 16, p);
                };
                float h[4] = {MINUS_INF, MINUS_INF, MINUS_INF, MINUS_INF};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (count > 0) weights(w);             // (there is no maximum before the first block)
#pragma unroll
                    for (int v = 2 * w; v < 2 * w + 2; ++v)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) h[e / 2 & 3] = fmaxf(h[e / 2 & 3], fmaxf(__uint_as_float(z[v][e]), __uint_as_float(z[v][e + 1])));
                }
                const float high = fmaxf(fmaxf(h[0], h[1]), fmaxf(h[2], h[3])) * a.scale_log2;
                if (count == 0 || __any_sync(0xffffffffu, high > top - a.room)) {
                    const float now = high > top - a.room ? high + a.headroom : top, keep = ex2_approx(top - now);
                    top = now;
                    sum = mul2(sum, pack2(keep, keep));
                    if (count > 0) {                       // (the products so far have ended: the logits' came behind them)
#pragma unroll 1
                        for (int e = 0; e < D; e += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_at + e, o);
#pragma unroll
                            for (int u = 0; u < 16; ++u) o[u] = __float_as_uint(__uint_as_float(o[u]) * keep);
                            tmem_st16(o_at + e, o);
                        }
                    }
                    more = more2 = pack2(0.f, 0.f);
                    weights(0);
                    weights(1);
                }
                ++count;
                tmem_st_wait();
                tell(bar_p + 8 * x);
                weights(2);
                weights(3);
                sum = add2(sum, add2(more, more2));
                tmem_st_wait();
                tell(bar_p2 + 8 * x);
            }
            if (!ok) break;
            // ---- the output
            const float2 both = unpack2(sum);
            const float total = both.x + both.y;
            if (count > 0) {
                ok = waited(bar_o + 8 * x, phase_o);
                if (!ok) break;
                phase_o ^= 1;
                tc_fence_after();
            }
            const bool none = total == 0.f, alone = k.ctas == 1;
            const float inv = none ? 0.f : 1.f / total;
            const int hq = it.h * R + r, t = it.t0 + x * tokens + tl;
            const bool there = tl < tokens && t < it.queries;
            __nv_bfloat16* const out = a.io.out + it.b * a.io.out_at[0] + hq * a.io.out_at[1] + t * a.io.out_at[2];
            const bool odd = any_bad[n & 1] != 0;
            float* const part = reinterpret_cast<float*>(smem) + (x * kTile + row) * S::kPitch;
            if (!alone) {
                // parts go where operands were: the other tile's products have to have ended too
                bool other = false;
                for (int i = it.k0; i < it.k1; ++i) {
                    const Columns c = it.tiles[x ^ 1].columns(it.blocks, i);
                    other |= c.lo != c.hi;
                }
                // (one item a CTA: its first output)
                ok = !other || waited(bar_o + 8 * (x ^ 1), 0);
                if (!ok) break;
                reinterpret_cast<float*>(smem + S::kPartEnds)[x * kTile + row] = top;
                reinterpret_cast<float*>(smem + S::kPartEnds)[2 * kTile + x * kTile + row] = total;
            } else if (a.lse && there) {
                a.lse[((int64_t)it.b * a.Hq + hq) * a.Tq + t] = none ? MINUS_INF : (top + log2f(total)) * kLn2;
            }
#pragma unroll 1
            for (int e = 0; e < D; e += 32) {
                uint32_t o[32];
                __syncwarp();
                if (count > 0) {
                    tmem_ld32_issue(o_at + e, o);
                    tmem_ld_wait();
                    pin32(o);
                } else {
#pragma unroll
                    for (int u = 0; u < 32; ++u) o[u] = 0;
                }
                if (odd && there) {
                    const Seen<TREE> sees = seen_by_row();
                    float extra[32] = {};
                    add_taken_out<D, TREE>(a, it, sees, bad + (n & 1) * kMasked * 4, hq, t, e, top, extra);
#pragma unroll
                    for (int u = 0; u < 32; ++u) o[u] = __float_as_uint(__uint_as_float(o[u]) + extra[u]);
                }
                if (!alone) {
#pragma unroll
                    for (int u = 0; u < 32; u += 4) *reinterpret_cast<uint4*>(part + e + u) = make_uint4(o[u], o[u + 1], o[u + 2], o[u + 3]);
                } else if (there) {
                    uint32_t p[16];
#pragma unroll
                    for (int u = 0; u < 16; ++u) p[u] = none ? 0u : bf16x2(__uint_as_float(o[2 * u]) * inv, __uint_as_float(o[2 * u + 1]) * inv);
                    if (k.wide) {
#pragma unroll
                        for (int u = 0; u < 16; u += 8)
                            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + e + 2 * u), "r"(p[u]), "r"(p[u + 1]), "r"(p[u + 2]),
                                         "r"(p[u + 3]), "r"(p[u + 4]), "r"(p[u + 5]), "r"(p[u + 6]), "r"(p[u + 7]) : "memory");
                    } else {
#pragma unroll
                        for (int u = 0; u < 16; u += 4) *reinterpret_cast<uint4*>(out + e + 2 * u) = make_uint4(p[u], p[u + 1], p[u + 2], p[u + 3]);
                    }
                }
            }
            if (count > 0) tell(bar_o_free + 8 * x);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_done + 8 * (n & 1));
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------------ tensor copies
            const auto waited = [&](uint32_t bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, k.limit_of(kRoleLoad)); };
            uint32_t slot = 0, phase = 0;
            int n = 0;
            bool ok = *abort_flag == 0;                    // (operands that lie nowhere are not fetched)
            const auto fetch = [&](const CUtensorMap* map, int row, int h, int b) {        // an operand to the ring
                if (!waited(bar_empty + 8 * slot, phase ^ 1)) return false;
                if (lane == 0) {
                    mbar_expect_tx(bar_full + 8 * slot, S::kOperand);
#pragma unroll
                    for (int i = 0; i < kSubs; ++i) tma_load_4d(base + S::kRing + slot * S::kOperand + i * 16384, map, bar_full + 8 * slot, i * 64, row, h, b);
                }
                ++issued;
                if (++slot == (uint32_t)kSlots) {
                    slot = 0;
                    phase ^= 1;
                }
                return true;
            };
            // the rows of V in a slot that are no numbers become zeros; a lane has rows lane, lane + 32, ..
            const auto take_out = [&](uint32_t at, uint32_t parity, uint32_t* words) {
                if (!waited(bar_full + 8 * at, parity)) return false;
                uint8_t* const v = smem + S::kRing + at * S::kOperand;
                uint32_t found_any = 0;
#pragma unroll 1
                for (int w = 0; w < 4; ++w) {
                    uint8_t* const row = v + (w * 32 + lane) * 128;
                    uint32_t any = 0;
#pragma unroll
                    for (int e = 0; e < kSubs * 8; ++e) {      // (pieces in another order in each lane: eight lie in all banks)
                        const uint4 y = *reinterpret_cast<const uint4*>(row + (e / 8) * 16384 + ((e + lane) & 7) * 16);
                        any |= ((y.x & 0x7F807F80u) + 0x00800080u) | ((y.y & 0x7F807F80u) + 0x00800080u) | ((y.z & 0x7F807F80u) + 0x00800080u) |
                               ((y.w & 0x7F807F80u) + 0x00800080u);
                    }
                    const bool odd = (any & 0x80008000u) != 0; // (an exponent of ones carries into the sign's place)
                    if (odd)
                        for (int e = 0; e < kSubs * 8; ++e) *reinterpret_cast<uint4*>(row + (e / 8) * 16384 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
                    const uint32_t found = __ballot_sync(0xffffffffu, odd);
                    if (lane == 0) words[w] = found;
                    found_any |= found;
                }
                if (lane == 0 && found_any) any_bad[n & 1] = 1;
                fence_async_proxy();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_checked + 8 * at);
                return true;
            };
            const auto publish = [&](const Item& it) {
                if (n >= 2 && !waited(bar_done + 8 * (n & 1), ((n >> 1) - 1) & 1)) return false;
                if (lane == 0) {
                    *reinterpret_cast<Item*>(smem + S::kItems + (n & 1) * kItemBytes) = it;
                    any_bad[n & 1] = 0;
                    mbar_arrive(bar_item + 8 * (n & 1));
                }
                __syncwarp();
                return true;
            };
            // The last tokens first: in front of a full window they are the ones with the most to look at.  Of a padded batch the items that are there are
            // counted, where there is a lane a sample, so that every CTA has as many: 8 x up to 704 tokens 70.8 us, 78.7 without.  (Every other round
            // dealt out from the other end: 73.9.)
            const bool known = a.query_len && a.B <= 32 && k.ctas == 1;
            const int queries = known && lane < a.B ? sample_of(a, lane).queries : 0, hands = gridDim.x / k.ctas, hand = blockIdx.x / k.ctas;
            const auto begin_of = [&](int tile) { return (k.per_head - 1 - tile) * 2 * tokens; };
            int level = 0, in_front = 0;                   // tiles of a head, from its end, and the items in front of this one's
            uint32_t with = __ballot_sync(0xffffffffu, queries > begin_of(0));
            for (int round = 0; ok; ++round) {
                int i = round * hands + hand, tile, b, h;
                if (known) {
                    while (level < k.per_head && i - in_front >= __popc(with) * a.H) {
                        in_front += __popc(with) * a.H;
                        ++level;
                        with = __ballot_sync(0xffffffffu, level < k.per_head && queries > begin_of(level));
                    }
                    if (level >= k.per_head) break;
                    tile = level;
                    i -= in_front;
                    int nth = quotient(i, k.heads);
                    h = i - nth * a.H;
                    uint32_t left = with;
                    for (; nth > 0; --nth) left &= left - 1;
                    b = __ffs(left) - 1;
                } else {
                    if (i >= k.items) break;
                    const int bhs = a.B * a.H;
                    tile = i / bhs;
                    i -= tile * bhs;
                    b = quotient(i, k.heads);
                    h = i - b * a.H;
                }
                const int t0 = begin_of(tile);
                const Sample s = sample_of(a, b);
                if (t0 >= s.queries) continue;
                Item it;
                it.there = 1;
                it.b = b;
                it.h = h;
                it.t0 = t0;
                it.len = s.len;
                it.queries = s.queries;
                it.blocks = blocks_of<TREE>(a, s, t0, t0 + 2 * tokens - 1);
                for (int x = 0; x < 2; ++x) {
                    it.tiles[x].span = span_of<TREE>(a, s, t0 + x * tokens, t0 + (x + 1) * tokens - 1);
                    it.tiles[x].whole = whole_of<TREE>(it.blocks, it.tiles[x].span);
                }
                const int each = it.blocks.n / k.ctas, more = it.blocks.n - each * k.ctas;
                it.k0 = rank * each + min(rank, more);
                it.k1 = it.k0 + each + (rank < more ? 1 : 0);
                ok = publish(it);
                if (!ok) break;
                if (it.k0 == it.k1) {                      // (no copies: nothing would wait for them before their places are used for something else)
                    ++n;
                    continue;
                }
                ok = fetched == 0 || waited(bar_q_free, (fetched - 1) & 1);
                if (!ok) break;
                if (lane == 0)
                    for (int x = 0; x < 2; ++x) {
                        mbar_expect_tx(bar_q + 8 * x, tokens * R * 128 * kSubs);
#pragma unroll
                        for (int e = 0; e < kSubs; ++e)
                            tma_load_4d(base + S::kQ + x * S::kOperand + e * 16384, &map_q, bar_q + 8 * x, e * 64, h * R, t0 + x * tokens, b * k.q_b);
                    }
                ++fetched;
                int masked = 0;
                uint32_t v_slot = 0, v_phase = 0;
                for (int j = it.k0; ok && j <= it.k1; ++j) {
                    const uint32_t before = v_slot, before_phase = v_phase;
                    if (j < it.k1) {
                        const int row = it.blocks.end(j) - kBlock;
                        ok = fetch(&map_k, row, h * k.k_h, b * k.k_b);
                        v_slot = slot;
                        v_phase = phase;
                        ok = ok && fetch(&map_v, row, h * k.v_h, b * k.v_b);
                    }
                    // the block before, whose V is there by now or soon
                    if (ok && j > it.k0 && !(it.tiles[0].columns(it.blocks, j - 1).all && it.tiles[1].columns(it.blocks, j - 1).all)) {
                        if (masked >= kMasked) *abort_flag = 1;
                        ok = masked < kMasked && take_out(before, before_phase, bad + ((n & 1) * kMasked + masked) * 4);
                        ++masked;
                    }
                }
                ++n;
            }
            if (ok) {
                Item end;
                end.there = 0;
                publish(end);
            }
        } else if (warp == kMmaWarp) {
            // -------------------------------------------------------------- products
            // (one lane all the way: what it spends between two products the tensor cores may spend waiting)
            if (elected()) {
                const unsigned long long lim = k.limit_of(kRoleMma);
                const uint32_t idesc_s = umma_idesc_bf16(kTile, 0) | (a.sign ? 1u << 13 : 0u), idesc_o = umma_idesc_bf16(kTile, D) | 1u << 16;
                uint32_t slot = 0, phase = 0, phase_q = 0, phase_p[2] = {0, 0}, phase_checked = 0, outputs[2] = {0, 0};
                const auto waited = [&](uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, lim); };
                // S(x) = Q(x) K^T over columns c; O(x) += P(x) V over tokens c
                const auto first_product = [&](int x, uint32_t ring, const Columns& c) {
                    const uint64_t dq = umma_desc_k128(base + S::kQ + x * S::kOperand), dk = umma_desc_k128(ring + c.lo * 128);
                    const uint32_t d = tmem_s(x) + c.lo, idesc = idesc_s | (uint32_t)((c.hi - c.lo) >> 3) << 17;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) tc_mma_bf16(d, further(dq, (e / 4) * 1024 + (e % 4) * 2), further(dk, (e / 4) * 1024 + (e % 4) * 2), idesc, e > 0 ? 1u : 0u);
                    tc_commit(bar_s + 8 * x);
                };
                const auto second_product = [&](int x, uint32_t ring, int lo, int hi, bool begun) {
                    const uint64_t dv = umma_desc_mn128(ring);
                    if (hi - lo == kBlock / 2) {
#pragma unroll
                        for (int e = 0; e < kBlock / 32; ++e) tc_mma_bf16_ts(tmem_o(x), tmem_s(x) + lo / 2 + 8 * e, further(dv, lo * 8 + e * 128), idesc_o, begun || e > 0 ? 1u : 0u);
                    } else {
#pragma unroll 1
                        for (int e = lo / 16; e < hi / 16; ++e, begun = true) tc_mma_bf16_ts(tmem_o(x), tmem_s(x) + 8 * e, further(dv, e * 128), idesc_o, begun ? 1u : 0u);
                    }
                };
                bool ok = true;
                for (int n = 0; ok; ++n) {
                    ok = waited(bar_item + 8 * (n & 1), (n >> 1) & 1);
                    const Item& it = items[n & 1];
                    if (!ok || !it.there) break;
                    const int k0 = it.k0, k1 = it.k1;
                    const Whole whole[2] = {it.tiles[0].whole, it.tiles[1].whole};
                    if (k0 == k1) {
                        mbar_arrive(bar_done + 8 * (n & 1));
                        continue;
                    }
                    ok = waited(bar_q, phase_q) && waited(bar_q + 8, phase_q);
                    phase_q ^= 1;
                    bool begun[2] = {false, false};
                    Columns before[2] = {{0, 0, true}, {0, 0, true}};
#pragma unroll 1
                    for (int i = k0; ok && i <= k1; ++i) {
                        // block i - 1's second product, block i's first
                        const bool second = i > k0, first = i < k1;
                        uint32_t v_slot = slot;
                        if (second) {
                            ok = waited(bar_full + 8 * slot, phase);
                            if (ok && !(before[0].all && before[1].all)) {
                                ok = waited(bar_checked + 8 * slot, phase_checked >> slot & 1);
                                phase_checked ^= 1u << slot;
                            }
                            if (++slot == (uint32_t)kSlots) {
                                slot = 0;
                                phase ^= 1;
                            }
                        }
                        Columns now[2] = {{0, 0, true}, {0, 0, true}};
                        if (first) {
                            ok = ok && waited(bar_full + 8 * slot, phase);
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                now[x].hi = kBlock;
                                if (i < whole[x].first || i >= whole[x].end) now[x] = columns_of(it.blocks, i, it.tiles[x].span);
                            }
                        }
                        const uint32_t v_ring = base + S::kRing + v_slot * S::kOperand, k_ring = base + S::kRing + slot * S::kOperand;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const bool adds = second && before[x].lo != before[x].hi;
                            if (ok && adds) {
                                ok = waited(bar_p + 8 * x, phase_p[x]);
                                if (ok && !begun[x] && outputs[x] > 0) ok = waited(bar_o_free + 8 * x, (outputs[x] - 1) & 1);
                            }
                            if (!ok) break;
                            tc_fence_after();
                            if (adds) {
                                second_product(x, v_ring, before[x].lo, min(before[x].hi, kBlock / 2), begun[x]);
                                begun[x] |= before[x].lo < kBlock / 2;
                                ok = waited(bar_p2 + 8 * x, phase_p[x]);
                                if (!ok) break;
                                phase_p[x] ^= 1;
                                tc_fence_after();
                                second_product(x, v_ring, max(before[x].lo, kBlock / 2), before[x].hi, begun[x]);
                                begun[x] = true;
                            }
                            if (!first && begun[x]) tc_commit(bar_o + 8 * x);
                            if (second && x == 1) tc_commit(bar_empty + 8 * v_slot);
                            if (now[x].lo != now[x].hi) first_product(x, k_ring, now[x]);
                            before[x] = now[x];
                        }
                        if (!ok) break;
                        if (first) {
                            tc_commit(bar_empty + 8 * slot);
                            if (++slot == (uint32_t)kSlots) {
                                slot = 0;
                                phase ^= 1;
                            }
                        }
                        if (i == k1 - 1) tc_commit(bar_q_free);
                    }
                    outputs[0] += begun[0] ? 1 : 0;
                    outputs[1] += begun[1] ? 1 : 0;
                    if (ok) mbar_arrive(bar_done + 8 * (n & 1));
                }
                tc_commit(bar_drain);                      // (waited for below)
            }
            __syncwarp();
        }
    }
    __syncthreads();
    // Another role may have given up behind the last product: operands and tensor memory stay until all of them have completed.
    // The same goes for copies in flight.
    if (warp == kLoadWarp && lane == 0 && *abort_flag) {
        for (uint32_t i = 0; i < (uint32_t)kSlots && i < issued; ++i) {
            const uint32_t at = issued - 1 - i;
            mbar_drain(bar_full + 8 * (at % kSlots), (at / kSlots) & 1);
        }
        for (int x = 0; fetched > 0 && x < 2; ++x) mbar_drain(bar_q + 8 * x, (fetched - 1) & 1);
    }
    if (tid == 0) {
        mbar_drain(bar_drain, 0);
        if (blockIdx.x == 0) *a.status = kStatusInReports | (int)gridDim.x;
        report_gave_up(a.status, *abort_flag != 0);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (k.ctas == 1) return;
    // ---------------------------------------------------------------------- the cluster's parts: rows in turn to its CTAs
    cluster_sync_all();
    const int tile = (blockIdx.x / k.ctas) / (a.B * a.H), bh = (blockIdx.x / k.ctas) - tile * a.B * a.H, b = quotient(bh, k.heads), h = bh - b * a.H;
    const int t0 = (k.per_head - 1 - tile) * 2 * tokens;
    const Sample s = sample_of(a, b);
    if (t0 < s.queries) {
        // what each part of a row counts by (kNothing: none weighs anything, the output is 0 whatever the parts are), a thread a row; then the sums, a thread
        // four elements
        const int mine = 2 * kTile / k.ctas;
        const float* const ends = reinterpret_cast<const float*>(smem + S::kPartEnds);
        float* const counts = reinterpret_cast<float*>(smem + S::kPartCounts);         // [rows][CTAs]
        const auto query_of = [&](int row, int& t, int& hq) {
            const int y = row / kTile, rl = row - y * kTile, tl = quotient(rl, a.R);
            t = t0 + y * tokens + tl;
            hq = h * R + (rl - tl * R);
            return tl < tokens && t < s.queries;
        };
        if (tid < mine) {
            const int row = rank + k.ctas * tid;
            const uint32_t at = smem_u32(ends + row);
            float tops[kMostCtas], sums[kMostCtas], top = kNoLogit, total = 0.f;
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c) {
                tops[c] = c < k.ctas ? cluster_ld(cluster_map(at, c)) : kNoLogit;
                sums[c] = c < k.ctas ? cluster_ld(cluster_map(at, c) + 2 * kTile * 4) : 0.f;
            }
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c) top = fmaxf(top, tops[c]);
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c) {
                tops[c] = ex2_approx(tops[c] - top);
                total = fmaf(sums[c], tops[c], total);
            }
            const bool none = total == 0.f;
            const float inv = 1.f / total;
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c)
                if (c < k.ctas) counts[tid * k.ctas + c] = none ? kNothing : tops[c] * inv;
            int t, hq;
            if (query_of(row, t, hq) && a.lse) a.lse[((int64_t)b * a.Hq + hq) * a.Tq + t] = none ? MINUS_INF : (top + log2f(total)) * kLn2;
        }
        __syncthreads();
#pragma unroll 2
        for (int i = tid; i < mine * (D / 4); i += kThreads) {
            const int j = i / (D / 4), e = i % (D / 4) * 4, row = rank + k.ctas * j;
            int t, hq;
            if (!query_of(row, t, hq)) continue;
            const uint32_t at = base + (row * S::kPitch + e) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c) {
                if (c >= k.ctas) break;
                const float4 y = cluster_ld4(cluster_map(at, c));
                const float f = counts[j * k.ctas + c];
                v.x = fmaf(y.x, f, v.x);
                v.y = fmaf(y.y, f, v.y);
                v.z = fmaf(y.z, f, v.z);
                v.w = fmaf(y.w, f, v.w);
            }
            if (counts[j * k.ctas] == kNothing) v = make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<uint2*>(a.io.out + b * a.io.out_at[0] + hq * a.io.out_at[1] + t * a.io.out_at[2] + e) = make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
        }
    }
    cluster_sync_all();                                    // (the others may still be reading what this CTA has)
}

// Rows of 64 elements as operands: a map over (d, n1, n2, n3) with boxes of (64, box1, box2, 1).  A dimension of one has no stride to speak of.
struct Dim {
    int64_t n, stride;
};
bool rows_map(CUtensorMap* map, const void* data, int d, Dim x1, Dim x2, Dim x3, int box1, int box2) {
    const Dim dims[3] = {x1, x2, x3};
    uint64_t n[4] = {(uint64_t)d}, bytes[3];
    for (int i = 0; i < 3; ++i) {
        n[i + 1] = (uint64_t)dims[i].n;
        bytes[i] = (uint64_t)(dims[i].n == 1 ? d : dims[i].stride) * 2;
    }
    const uint32_t box[4] = {64, (uint32_t)box1, (uint32_t)box2, 1};
    return make_bf16_map_4d(map, data, n, bytes, box);
}

template <int D, bool TREE>
int launch_tiles(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const TilesArgs& k, int grid, cudaStream_t stream) {
    static DoneOnDevice done;
    const int rc = allow_dynamic_smem(attention_tiles_kernel<D, TREE>, TilesSmem<D>::kBytes, done);
    if (rc != VITCOP_OK) return rc;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)k.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = TilesSmem<D>::kBytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 2 : 1;
    KernelTimeScope timed("attention_tiles_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, attention_tiles_kernel<D, TREE>, mq, mk, mv, k));
}

// Clusters of this size that run at a time, an SM a CTA (all kernels of this file alike): not SMs / ctas, for a cluster stays inside a group of SMs.
int clusters_that_run(int ctas) {
    static KnownOnDevice known[3];
    static DoneOnDevice done;
    constexpr int kBytes = TilesSmem<128>::kBytes;
    const auto allow = [] { return allow_dynamic_smem(attention_tiles_kernel<128, false>, kBytes, done); };
    return clusters_at_once(attention_tiles_kernel<128, false>, ctas, kThreads, kBytes, allow, known[ctas == 2 ? 0 : ctas == 4 ? 1 : 2]);
}

}  // namespace

// How a call is shared out, and about how many us that takes: items have a beginning and an end of 5 (a kernel's first 11), a block of two tiles 1.9 and of one
// 1.6; a cluster's join 3.  Clusters that do not all run at once take twice as long: 16 to 18 items of 1500 rows 35.5 us in eights, 20.9 in fours; 34 to 37 39.2 in fours,
// 26.7 in pairs (this B200 runs 15 clusters of eight and 33 of four).  Measured (estimate in brackets), in clusters of four and by the other kernel at its best: 64 rows of 32 heads of 128, 355 tokens
// 13.5 and 10.8 us (16), 1059 tokens 19.0 and 15.0 (18), 4195 tokens 29.4 and 31.1 (28); 256 rows, 1315 tokens 22.1 and 31.4 (20).  Items in turn: 512 of
// 256 rows, 547 tokens 70.7 and 197 (58); 256 of 256 rows, 547 tokens 35.2 and 104.7 (35), of heads of 64 30.1 and 60.1 (35).  Heads of 64 are 0 to 17 % faster than heads of 128, and no
// choice between the kernels hung on it: 64 rows of 64 heads, 4195 tokens 35.4 and 30.0 (40), 32 heads, 1500 tokens 17.2 and 21.2 (20), 300 rows of 32, 2000 tokens 25.9 and 47.4 (29).
// 64 tokens x 28 heads over 16512 rows, clusters of eight: 51 and 91 (45).
struct TilesPlan {
    int tokens, per_head, ctas;
    int64_t items;
    double us;
};
static TilesPlan tiles_plan(const SeqArgs& a, int d) {
    TilesPlan p = {0, 0, 1, 0, 1e30};
    const int R = (int)a.R.d;
    if (d == 256 || R > kTile / 2 || a.N == 0) return p;
    p.tokens = kTile / R;
    p.per_head = (a.Tq + 2 * p.tokens - 1) / (2 * p.tokens);
    p.items = (int64_t)a.B * a.H * p.per_head;
    if (p.items > 0x7fffffff / kMostCtas) return p;
    // tokens that an item's rows may see
    int64_t span = a.N;
    if (!a.tree) span = std::min<int64_t>(span, (int64_t)a.n_sink + a.window + std::min(a.Tq, 2 * p.tokens));
    const int64_t blocks = (span + kBlock - 1) / kBlock;
    const int sms = std::min(sm_count(), kMaxReports);
    while (p.ctas < kMostCtas && p.items * p.ctas * 2 <= sms && p.ctas * 2 <= blocks && p.items <= clusters_that_run(p.ctas * 2)) p.ctas *= 2;
    const double block = a.Tq > p.tokens ? 1.9 : 1.6;
    p.us = p.items <= sms ? 11 + block * blocks / p.ctas + (p.ctas > 1 ? 3 : 0) : 6 + std::ceil((double)p.items / sms) * (5 + block * blocks);
    return p;
}
double tiles_kernel_us(const SeqArgs& a, int d) { return tiles_plan(a, d).us; }

// ERR_UNSUPPORTED where rows lie so that tensor copies cannot fetch them.
int launch_attention_tiles(const SeqArgs& a, int d, cudaStream_t stream) {
    TilesArgs k;
    k.a = a;
    const SeqRows& io = a.io;
    const int R = (int)a.R.d;
    const TilesPlan plan = tiles_plan(a, d);
    k.tokens = plan.tokens;
    k.per_head = plan.per_head;
    k.items = (int)plan.items;
    k.ctas = plan.ctas;
    k.heads = divisor(a.H);
    const auto step = [](int n, int64_t stride) { return n > 1 && stride == 0 ? 0 : 1; };
    k.q_b = step(a.B, io.q_at[0]);
    k.k_b = step(a.B, io.k_at[0]);
    k.k_h = step(a.H, io.k_at[1]);
    k.v_b = step(a.B, io.v_at[0]);
    k.v_h = step(a.H, io.v_at[1]);
    if (!step(a.Hq, io.q_at[1]) || !step(a.Tq, io.q_at[2]) || !step(a.N, io.k_at[2]) || !step(a.N, io.v_at[2])) return VITCOP_ERR_UNSUPPORTED;
    CUtensorMap mq, mk, mv;
    if (!rows_map(&mq, io.q, d, {a.Hq, io.q_at[1]}, {a.Tq, io.q_at[2]}, {k.q_b ? a.B : 1, io.q_at[0]}, R, k.tokens) ||
        !rows_map(&mk, io.K, d, {a.N, io.k_at[2]}, {k.k_h ? a.H : 1, io.k_at[1]}, {k.k_b ? a.B : 1, io.k_at[0]}, kBlock, 1) ||
        !rows_map(&mv, io.V, d, {a.N, io.v_at[2]}, {k.v_h ? a.H : 1, io.v_at[1]}, {k.v_b ? a.B : 1, io.v_at[0]}, kBlock, 1))
        return VITCOP_ERR_UNSUPPORTED;
    k.wide = reinterpret_cast<uintptr_t>(io.out) % 32 == 0 && io.out_at[0] % 16 == 0 && io.out_at[1] % 16 == 0 && io.out_at[2] % 16 == 0;
    k.wait_ns = gram_wait_limit_ns();
    k.expire_roles = pair_expire_roles();
    const int sms = std::min(sm_count(), kMaxReports), grid = (int)(k.ctas > 1 ? plan.items * k.ctas : std::min<int64_t>(plan.items, sms));
    if (d == 64) return a.tree ? launch_tiles<64, true>(mq, mk, mv, k, grid, stream) : launch_tiles<64, false>(mq, mk, mv, k, grid, stream);
    return a.tree ? launch_tiles<128, true>(mq, mk, mv, k, grid, stream) : launch_tiles<128, false>(mq, mk, mv, k, grid, stream);
}

}  // namespace vitcop
