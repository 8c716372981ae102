// Attention of query rows over the K/V cache in 4 bits: out = softmax(scale q K^T) V over the rows that a query sees.
//
// Every product is one of matrix instructions (m16n8k16, bf16 in, fp32 out), and codes become operands in registers:
//   logits   tokens times query rows (Hq / H heads times Tq queries, a tile of 8 NT of them at a time).  A code c is the bf16
//            128 + c (its nibble under the exponent of 128), exactly; per group the token's scale multiplies the product in fp32.
//            The centres, and the scales times -136, are one more product each, with the groups' sums of q split into three bf16
//   output   elements times query rows: (128 + c) - 136 = c - 8 is exact too.  The weights enter, transposed, as bf16(p) with the
//            centres and as bf16(bf16(p) s) with a group's codes; what the output is divided by is the sum of the bf16(p) (rows of ones
//            beside the centres), so that a row that takes nearly all is not off by its weight's rounding
// What is rounded, and why: the matrix instructions take operands of 16 bits.  Weights are bf16, which holds 2^-100 of a row's largest as it
// holds the largest; fp16 (three bits more) would need a power of two for every row and group.  Weight times scale is the operand in
// place of the scaled code, which would cost a product for each of a block's elements instead of one for each of its groups.  Together they add 0.001 to the
// 0.0016 that the output's own rounding to bf16 is off by (root mean square against 64 bits: 0.0018 to 0.0020).  128 + c in place of c costs the
// logits' fp32 sums some five bits, and saves an instruction for every two codes of K.
// A warp takes every fourth (or eighth) block of 32 tokens of its CTA's piece, with blocks ahead in shared memory (cp.async), and keeps
// maximum, sum and output of its own; the CTA joins its warps, a second kernel joins the CTAs that shared a head.
// Bound by instructions: 680 a block (d = 128, eight rows or fewer), most of them what turns four bits into operands, which the ALU pipe
// takes every second cycle.  16 x 32 heads of 128, one query each: 2048 tokens 44 us, 3.8 TB/s of cache (the copy rate is 6.5), 4096
// tokens 4.2 TB/s; issue slots 58 %, ALU 57 %, tensor pipe 26 %.  256 tokens of 32 heads: 4.9 us, of which the launch is more than half.
#include <type_traits>

#include "async_copy.cuh"
#include "kv_attention.cuh"

namespace vitcop {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = 2;
constexpr uint32_t kOnes = 0x3F803F80u;                    // 1, twice, in bf16
constexpr int kWholeBlocks = 24;                           // what pieces of heads cost at least, in blocks of a CTA
// Weights are 2^(logit - base) with a base that starts this far above the maximum: they stay below 2^-16, so that sums of weights times
// values of V hold wherever those values lie in fp32's range, and the smallest that count are still 2^-100 of the largest.
constexpr float kHeadroom = 24.f;

// Resident CTAs an SM, which the registers of the accumulators and the ring's memory leave room for.
constexpr int ctas_per_sm(int D, int NT) { return D == 256 || D * NT > 256 ? 2 : D * NT <= 128 ? 4 : 3; }

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// d = a b
__device__ __forceinline__ void mma_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // an 8 x 8 matrix of 16-bit values, two of a row in a lane
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int BYTES>
__device__ __forceinline__ void lds(uint32_t* w, const uint8_t* p) {
    if constexpr (BYTES >= 16) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(p + 16 * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    } else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// Eight query rows as operand, one lane's part: its eight elements of each group of row g, and the groups' sums in three bf16 each
// (part p of group i is element p G + i of the products with centres and scales).
template <int G>
struct __align__(16) QueryOperand {
    uint4 q[G];
    uint4 sums;                                            // (the second half: eight groups)
};
template <int G>
__device__ __forceinline__ void make_operand(QueryOperand<G>* to, const uint4* raw, uint32_t sign, int t) {
    float total[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
        uint4 v = raw[i * 32];
        v = make_uint4(v.x ^ sign, v.y ^ sign, v.z ^ sign, v.w ^ sign);
        // elements 0 and 4, 1 and 5, 2 and 6, 3 and 7, as the codes lie
        to->q[i] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
        float x = ((bf16lo(v.x) + bf16hi(v.x)) + (bf16lo(v.y) + bf16hi(v.y))) + ((bf16lo(v.z) + bf16hi(v.z)) + (bf16lo(v.w) + bf16hi(v.w)));
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        total[i] = x;
    }
    uint32_t sums[4] = {};
#pragma unroll
    for (int i = 0; i < (G == 8 ? 4 : 2); ++i) {
        float v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int k = 2 * t + 8 * i + e, p = k / G;
            float x = 0.f;
#pragma unroll
            for (int j = 0; j < G; ++j)
                if (k % G == j) x = total[j];
            const float first = __bfloat162float(__float2bfloat16_rn(x)), second = __bfloat162float(__float2bfloat16_rn(x - first));
            v[e] = p == 0 ? first : p == 1 ? second : p == 2 ? (x - first) - second : 0.f;
        }
        sums[i] = bf16x2(v[0], v[1]);
    }
    to->sums = make_uint4(sums[0], sums[1], sums[2], sums[3]);
}

// Where a CTA is in its share of the work: block `tile` of segment `seg` (head and tile of rows) of sample b, `left` blocks to go.
struct Walk {
    int b, seg, tile, blocks, left, len;                   // (len: of a CTA without a share)
};
__device__ __forceinline__ int len_of(const AttArgs& a, int b) { return a.cache_len ? max(0, min(__ldcg(a.cache_len + b), a.Ncap)) : a.Ncap; }
__device__ __forceinline__ int blocks_of(const AttArgs& a, int b) { return (len_of(a, b) + kCacheBlock - 1) / kCacheBlock; }
// How `total` blocks are shared out: the first `more` of `ctas` CTAs have `each` + 1 blocks, the others `each`; `whole`: a CTA has
// the blocks of one segment instead.
struct Shares {
    int ctas, each, more;
    bool whole;
};
__device__ __forceinline__ Shares shares_of(int total, int longest, int segs, int most) {
    Shares s;
    // as few as take no more rounds of a block a warp than all of them would: fewer pieces, and every warp has work in the last round
    const int rounds = max(1, (total + most * kWarps - 1) / (most * kWarps));
    s.ctas = rounds > 2 ? most : max(1, (total + rounds * kWarps - 1) / (rounds * kWarps));
    s.each = total / s.ctas;
    s.more = total - s.each * s.ctas;
    // where the longest segment takes hardly longer than a fair share, pieces to join and heads to begin anew cost more
    s.whole = segs <= most && longest <= s.each + kWholeBlocks;
    return s;
}
__device__ __forceinline__ int first_of(const Shares& s, int cta) { return cta * s.each + min(cta, s.more); }
__device__ __forceinline__ int holder_of(const Shares& s, int block) {
    const int front = s.more * (s.each + 1);
    return block < front ? block / (s.each + 1) : s.more + (block - front) / s.each;
}
__device__ __forceinline__ int piece(const Walk& w) { return min(w.blocks - w.tile, w.left); }

// SHARES: the blocks of all heads are shared out to the CTAs; otherwise a CTA has a head and tile of rows.  W: warps of a CTA.
template <int D, int NT, bool SHARES, int W>
__global__ void __launch_bounds__(W * 32, ctas_per_sm(D, NT) * kWarps / W > 0 ? ctas_per_sm(D, NT) * kWarps / W : 1)
cache_attention_kernel(AttArgs a) {
    static_assert(!SHARES || W == kWarps, "shares are counted in rounds of kWarps blocks");
    using L = CacheBlock<D>;
    constexpr int G = L::G, NR = 8 * NT;
    constexpr int kChunks = L::kBytes / 16;
    extern __shared__ __align__(128) uint8_t smem[];
    float* const join = reinterpret_cast<float*>(smem + W * kStages * L::kBytes);      // [warp][2 groups][8][lane]
    float* const join_max = join + W * 512;                                            // [warp][NR]
    float* const join_sum = join_max + W * NR;
    float* const join_weight = join_sum + W * NR;
    QueryOperand<G>* const operand = reinterpret_cast<QueryOperand<G>*>(join_weight + W * NR);      // [NT][lane]
    uint4* const queries = reinterpret_cast<uint4*>(operand + NT * 32);                                // [stage][NT][G][lane]
    Walk* const walks = reinterpret_cast<Walk*>(queries + kStages * NT * G * 32);                                   // [warp][2]
    int32_t* const stage_at = reinterpret_cast<int32_t*>(walks + W * 2);                         // of warp 0
    int32_t* const before = stage_at + 1;                           // [B + 2], and the samples' lengths [B]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int segs = a.H * a.RT.d;
    grid_dependency_wait();
    if constexpr (SHARES) grid_dependency_launch_dependents();     // (the join's CTAs, which wait for this grid to end)
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = VITCOP_OK;

    // (kept in shared memory, one copy a warp: registers are what the blocks' work is short of)
    Walk* const at_work = walks + warp * 2;
    Walk* const at_fetch = walks + warp * 2 + 1;
    Walk now;
    if constexpr (SHARES) {
        // blocks in front of each sample, and of the longest
        if (warp == 0) {
            int sum = 0, longest = 0;
            for (int b0 = 0; b0 < a.B; b0 += 32) {
                const int len = b0 + lane < a.B ? len_of(a, b0 + lane) : 0;
                int v = (len + kCacheBlock - 1) / kCacheBlock;
                const int mine = v;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, v, off);
                    if (lane >= off) v += u;
                }
                if (b0 + lane < a.B) {
                    before[b0 + lane] = sum + v - mine;
                    before[a.B + 2 + b0 + lane] = len;
                }
                sum += __shfl_sync(0xffffffffu, v, 31);
                longest = max(longest, mine);
            }
            longest = __reduce_max_sync(0xffffffffu, longest);
            if (lane == 0) {
                before[a.B] = sum;
                before[a.B + 1] = longest;
            }
        }
        __syncthreads();
        const int total = before[a.B] * segs;
        const Shares share = shares_of(total, before[a.B + 1], a.B * segs, gridDim.x);
        if (share.whole) {
            if ((int)blockIdx.x >= a.B * segs) return;
            now.b = blockIdx.x / segs;
            now.seg = blockIdx.x - now.b * segs;
            now.tile = 0;
            now.blocks = now.left = before[now.b + 1] - before[now.b];
        } else {
            if ((int)blockIdx.x >= share.ctas || total == 0) return;
            const int from = first_of(share, blockIdx.x);
            int lo = 0, hi = a.B;                          // the last sample that starts at or before `from`: it has blocks
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (before[mid] * segs <= from) lo = mid; else hi = mid;
            }
            now.b = lo;
            now.blocks = before[lo + 1] - before[lo];
            const int in = from - before[lo] * segs;
            now.seg = in / now.blocks;
            now.tile = in - now.seg * now.blocks;
            now.left = first_of(share, blockIdx.x + 1) - from;
        }
    } else {
        now.b = blockIdx.x / segs;
        now.seg = blockIdx.x - now.b * segs;
        now.tile = 0;
        now.len = len_of(a, now.b);
        now.blocks = now.left = a.Ncap / kCacheBlock;      // (as long as the length is on its way)
    }
    const auto next = [&](Walk& w) {                       // to the piece behind
        w.left -= piece(w);
        w.tile = 0;
        if (++w.seg == segs) {
            w.seg = 0;
            if constexpr (SHARES)
                if (w.left > 0) do { ++w.b; w.blocks = before[w.b + 1] - before[w.b]; } while (w.blocks == 0);
        }
    };
    // (a walk is copied, and written back by one lane, between barriers of the warp)
    const auto put = [&](Walk* to, const Walk& w) {
        __syncwarp();
        if (lane == 0) *to = w;
        __syncwarp();
    };
    // the sequence's blocks ahead of their use: this warp's share of every piece
    const auto first_block = [&](const Walk& w) {
        return a.cache + (((int64_t)w.b * a.H + quotient(w.seg, a.RT)) * (a.Ncap / kCacheBlock) + w.tile + warp) * L::kBytes + lane * 16;
    };
    if constexpr (SHARES) put(at_work, now);
    put(at_fetch, now);
    int ahead_left = piece(now) - warp;                    // blocks of the piece from this warp's next on
    const uint8_t* ahead_src = first_block(now);
    uint8_t* const ring = smem + warp * kStages * L::kBytes;
    const uint32_t ring_at = smem_u32(ring) + lane * 16;
    int fill = 0;
    bool begins = true;                                    // a piece, whose queries come with its first block
    const auto fetch = [&]() {
        if (SHARES && ahead_left <= 0) {
            Walk w = *at_fetch;
            while (ahead_left <= 0 && w.left > piece(w)) {
                next(w);
                ahead_left = piece(w) - warp;
                ahead_src = first_block(w);
                begins = true;
            }
            put(at_fetch, w);
        }
        if (ahead_left > 0) {
            const uint32_t dst = ring_at + fill * L::kBytes;
#pragma unroll
            for (int i = 0; i < kChunks / 32; ++i)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i * 512), "l"(ahead_src + i * 512) : "memory");
            if (warp == 0 && begins) {
                begins = false;
                const int b = at_fetch->b, seg = at_fetch->seg, h = quotient(seg, a.RT), row0 = (seg - h * (int)a.RT.d) * NR;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int r = row0 + n * 8 + g, tq = quotient(r, a.R), hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
                    const bool there = r < (int)a.R.d * a.Tq;
                    const __nv_bfloat16* const src = a.io.q + (there ? b * a.io.qb + hq * a.io.qh + tq * a.io.qt + t * 8 : 0);
                    const uint32_t to = smem_u32(queries + ((fill * NT + n) * G) * 32 + lane);
#pragma unroll
                    for (int i = 0; i < G; ++i)            // (rows behind the last are zeros)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * 512), "l"(src + (there ? i * 32 : 0)), "r"(there ? 16 : 0)
                                     : "memory");
                }
            }
            ahead_left -= W;
            ahead_src += W * L::kBytes;
            fill = fill + 1 == kStages ? 0 : fill + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) fetch();
    if constexpr (!SHARES) {                               // the first blocks have not waited for it
        now.blocks = now.left = (now.len + kCacheBlock - 1) / kCacheBlock;
        ahead_left += now.blocks - a.Ncap / kCacheBlock;
        put(at_work, now);
    }
    int use = 0;

    do {
        now = *at_work;
        const int b = now.b, h = quotient(now.seg, a.RT), row0 = (now.seg - h * (int)a.RT.d) * NR, rows = (int)a.R.d * a.Tq;
        const int count = piece(now);
        const int len = SHARES ? before[a.B + 2 + b] : now.len;
        // (they came with the first block of warp 0)
        if (warp == 0) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            if (NT > 1 && lane == 0) *stage_at = use;
        }
        if constexpr (NT > 1) __syncthreads(); else __syncwarp();
        if (warp < NT) {
            const int at = NT > 1 ? *stage_at : use;
            make_operand<G>(operand + warp * 32 + lane, queries + ((at * NT + warp) * G) * 32 + lane, a.sign, t);
        }
        // o[n][i][j][e]: element i 32 + 4 g + 2 j + e / 2 of row n 8 + 2 t + e % 2; base, sum: rows n 8 + 2 t + e, in powers of two
        float o[NT][G][2][4], oc[NT][4], base[NT][2], sum[NT][2];
        int limit[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = row0 + n * 8 + 2 * t + e;
                limit[n][e] = r < rows ? (a.causal ? max(0, len - a.Tq + quotient(r, a.R) + 1) : len) : 0;
                base[n][e] = kNoLogit;
                sum[n][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                oc[n][e] = 0.f;
#pragma unroll
                for (int i = 0; i < G; ++i) o[n][i][0][e] = o[n][i][1][e] = 0.f;
            }
        }
        // (rows are ordered by query: the first sees least, the last most)
        const int last = min(row0 + NR, rows) - 1;
        const int least = a.causal ? max(0, len - a.Tq + quotient(row0, a.R) + 1) : len;
        const int most = a.causal ? max(0, len - a.Tq + quotient(last, a.R) + 1) : len;

        // Half m of a block: 16 tokens from token0 on.  z[n][e]: token g + 8 (e / 2), row n 8 + 2 t + e % 2.  EDGE: some row does not
        // see some of them.
        const auto half_block = [&](const uint8_t* block, int m, int token0, auto edge_) {
            constexpr bool EDGE = decltype(edge_)::value;
            float z[NT][4];
            {
                const int r = 16 * m + g;
                uint32_t k0[G], k1[G], s0[(G + 1) / 2], s1[(G + 1) / 2];
                lds<4 * G>(k0, block + L::kKCodes + r * (D / 2) + t * 4 * G);
                lds<4 * G>(k1, block + L::kKCodes + (r + 8) * (D / 2) + t * 4 * G);
                lds<2 * G>(s0, block + L::kKScale + r * 2 * G);
                lds<2 * G>(s1, block + L::kKScale + (r + 8) * 2 * G);
                const int pair = 2 * ((2 * t) % G);
                const uint32_t c0 = *reinterpret_cast<const uint32_t*>(block + L::kKCentre + r * 2 * G + pair);
                const uint32_t c1 = *reinterpret_cast<const uint32_t*>(block + L::kKCentre + (r + 8) * 2 * G + pair);
                const uint32_t f0 = *reinterpret_cast<const uint32_t*>(block + L::kKScale + r * 2 * G + pair);
                const uint32_t f1 = *reinterpret_cast<const uint32_t*>(block + L::kKScale + (r + 8) * 2 * G + pair);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 u = operand[n * 32 + lane].sums;
                    float f[4];
                    mma_zero(z[n], c0, c1, c0, c1, u.x, u.y);
                    mma_zero(f, f0, f1, f0, f1, u.x, u.y);
                    if constexpr (G == 8) {
                        mma(z[n], c0, c1, c0, c1, u.z, u.w);
                        mma(f, f0, f1, f0, f1, u.z, u.w);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[n][e] = fmaf(-136.f, f[e], z[n][e]);
                }
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    uint32_t x0[4], x1[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x0[e] = code_pair(k0[i] >> (4 * e));
                        x1[e] = code_pair(k1[i] >> (4 * e));
                    }
                    const float h0 = i & 1 ? bf16hi(s0[i / 2]) : bf16lo(s0[i / 2]), h1 = i & 1 ? bf16hi(s1[i / 2]) : bf16lo(s1[i / 2]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 u = operand[n * 32 + lane].q[i];
                        float acc[4];
                        mma_zero(acc, x0[0], x1[0], x0[1], x1[1], u.x, u.y);
                        mma(acc, x0[2], x1[2], x0[3], x1[3], u.z, u.w);
                        z[n][0] = fmaf(h0, acc[0], z[n][0]);
                        z[n][1] = fmaf(h0, acc[1], z[n][1]);
                        z[n][2] = fmaf(h1, acc[2], z[n][2]);
                        z[n][3] = fmaf(h1, acc[3], z[n][3]);
                    }
                }
            }
            uint32_t p[NT][2], seen[NT][2];                // weights of tokens 2 t, 2 t + 1 and 8 behind, row n 8 + g; which of them it sees
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (EDGE) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (token0 + g + 8 * (e / 2) >= limit[n][e & 1]) z[n][e] = MINUS_INF;
                    const int even = __shfl_sync(0xffffffffu, limit[n][0], g >> 1), odd = __shfl_sync(0xffffffffu, limit[n][1], g >> 1);
                    const int there = (g & 1 ? odd : even) - token0 - 2 * t;
                    seen[n][0] = (there > 0 ? 0x0000FFFFu : 0u) | (there > 1 ? 0xFFFF0000u : 0u);
                    seen[n][1] = (there > 8 ? 0x0000FFFFu : 0u) | (there > 9 ? 0xFFFF0000u : 0u);
                }
                // (the sums stay relative to an older maximum until a logit has passed it by 2^8)
                float high[2] = {fmaxf(z[n][0], z[n][2]), fmaxf(z[n][1], z[n][3])};
                if (__any_sync(0xffffffffu, fmaf(high[0], a.scale_log2, -base[n][0]) > 8.f - kHeadroom || fmaf(high[1], a.scale_log2, -base[n][1]) > 8.f - kHeadroom)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) high[e] = fmaxf(high[e], __shfl_xor_sync(0xffffffffu, high[e], off));
                        const float top = fmaxf(base[n][e], fmaf(high[e], a.scale_log2, kHeadroom)), keep = ex2_approx(base[n][e] - top);
                        base[n][e] = top;
                        sum[n][e] *= keep;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            oc[n][2 * h + e] *= keep;
#pragma unroll
                            for (int i = 0; i < G; ++i) {
                                o[n][i][0][2 * h + e] *= keep;
                                o[n][i][1][2 * h + e] *= keep;
                            }
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[n][e] = ex2_approx(fmaf(z[n][e], a.scale_log2, -base[n][e & 1]));
                    sum[n][e & 1] += z[n][e];
                }
                p[n][0] = transposed(bf16x2(z[n][0], z[n][1]));
                p[n][1] = transposed(bf16x2(z[n][2], z[n][3]));
            }
            {
                const int v = m * 16 + 2 * t;              // tokens v, v + 1, v + 8, v + 9
                uint32_t w[4][(G + 1) / 2], s0[G], s1[G];
#pragma unroll
                for (int e = 0; e < 4; ++e) lds<2 * G>(w[e], block + L::kVCodes + (v + (e & 1) + 8 * (e / 2)) * (D / 2) + g * 2 * G);
                lds<4 * G>(s0, block + L::kVScale + v * 2 * G);
                lds<4 * G>(s1, block + L::kVScale + (v + 8) * 2 * G);
                uint32_t c0 = *reinterpret_cast<const uint32_t*>(block + L::kVCentre + ((g % G) * 32 + v) * 2);
                uint32_t c1 = *reinterpret_cast<const uint32_t*>(block + L::kVCentre + ((g % G) * 32 + v + 8) * 2);
                if (g >= G) c0 = c1 = 0u;
                if constexpr (EDGE) {                      // (what nobody wrote may be no number; what was written is one)
                    const int there = len - token0 - 2 * t;
                    c0 &= (there > 0 ? 0x0000FFFFu : 0u) | (there > 1 ? 0xFFFF0000u : 0u);
                    c1 &= (there > 8 ? 0x0000FFFFu : 0u) | (there > 9 ? 0xFFFF0000u : 0u);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) mma(oc[n], c0, kOnes, c1, kOnes, p[n][0], p[n][1]);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
                    const uint32_t lo = __byte_perm(w[0][i / 2], w[1][i / 2], pick), hi = __byte_perm(w[2][i / 2], w[3][i / 2], pick);
                    const uint32_t f0 = __byte_perm(s0[i / 2], s0[(G + i) / 2], pick), f1 = __byte_perm(s1[i / 2], s1[(G + i) / 2], pick);
                    uint32_t x[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = centred(code_pair(lo >> (4 * e)));
                        x[4 + e] = centred(code_pair(hi >> (4 * e)));
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t b0 = times(p[n][0], f0), b1 = times(p[n][1], f1);
                        if constexpr (EDGE) {              // (the scale of a row that this query does not see may be no number)
                            b0 &= seen[n][0];
                            b1 &= seen[n][1];
                        }
                        mma(o[n][i][0], x[0], x[1], x[4], x[5], b0, b1);
                        mma(o[n][i][1], x[2], x[3], x[6], x[7], b0, b1);
                    }
                }
            }
        };

        __syncthreads();                                   // (the queries)
        int token0 = (now.tile + warp) * kCacheBlock;
        for (const int end = (now.tile + count) * kCacheBlock; token0 < end; token0 += W * kCacheBlock) {
            const uint8_t* const block = ring + use * L::kBytes;
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();
#pragma unroll 1
            for (int m = 0; m < 2; ++m) {
                const int token = token0 + 16 * m;
                if (token + 16 <= least) half_block(block, m, token, std::false_type{});
                else if (token < most) half_block(block, m, token, std::true_type{});
            }
            __syncwarp();
            fetch();
            use = use + 1 == kStages ? 0 : use + 1;
        }

        // the CTA's warps joined, two groups at a time
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], off);
                if (g == 0) {
                    join_max[warp * NR + n * 8 + 2 * t + e] = base[n][e];
                    join_sum[warp * NR + n * 8 + 2 * t + e] = sum[n][e];
                    join_weight[warp * NR + n * 8 + 2 * t + e] = oc[n][2 + e];       // (rows 8 to 15 are all the sum of the weights)
                }
            }
        now = *at_work;
        const bool whole = now.tile == 0 && count == now.blocks;
        float* const part = SHARES && !whole ? a.part + (size_t)(2 * blockIdx.x + (now.tile == 0 ? 1 : 0)) * NR * (D + 3) : nullptr;
        const int je = warp & 1, ji = warp >> 1 & 1;       // this warp's share (of the first four): group i0 + ji, rows n 8 + 2 t + je
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int rl = n * 8 + 2 * t + je, r = row0 + rl;
            float f[W], high = kNoLogit, total = 0.f, weight = 0.f;
#pragma unroll
            for (int i0 = 0; i0 < G; i0 += 2) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float c = __shfl_sync(0xffffffffu, oc[n][e], 4 * (i0 + i) + t);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            join[((warp * 2 + i) * 8 + 4 * e + 2 * j) * 32 + lane] = o[n][i0 + i][j][e] + c;
                            join[((warp * 2 + i) * 8 + 4 * e + 2 * j + 1) * 32 + lane] = o[n][i0 + i][j][2 + e] + c;
                        }
                    }
                __syncthreads();
                if (i0 == 0) {
#pragma unroll
                    for (int w = 0; w < W; ++w) high = fmaxf(high, join_max[w * NR + rl]);
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        f[w] = ex2_approx(join_max[w * NR + rl] - high);
                        total = fmaf(join_sum[w * NR + rl], f[w], total);
                        weight = fmaf(join_weight[w * NR + rl], f[w], weight);
                    }
                }
                float v[4] = {};
#pragma unroll
                for (int w = 0; w < W; ++w)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = fmaf(join[((w * 2 + ji) * 8 + 4 * je + k) * 32 + lane], f[w], v[k]);
                const bool none = total == 0.f;
                const int tq = quotient(r, a.R), hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
                if (r < rows && warp < 4) {
                    if (part) {
                        *reinterpret_cast<float4*>(part + rl * D + (i0 + ji) * 32 + 4 * g) = make_float4(v[0], v[1], v[2], v[3]);
                        if (i0 == 0 && ji == 0 && g == 0) {
                            part[NR * D + rl] = high;
                            part[NR * D + NR + rl] = total;
                            part[NR * D + 2 * NR + rl] = weight;
                        }
                    } else {
                        const float inv = none ? 0.f : 1.f / weight;
                        *reinterpret_cast<uint2*>(a.io.out + b * a.io.ob + hq * a.io.oh + tq * a.io.ot + (i0 + ji) * 32 + 4 * g) =
                            make_uint2(bf16x2(v[0] * inv, v[1] * inv), bf16x2(v[2] * inv, v[3] * inv));
                        if (i0 == 0 && ji == 0 && g == 0 && a.lse)
                            a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = none ? MINUS_INF : (high + __log2f(total)) * kLn2;
                    }
                }
                __syncthreads();
            }
        }
        next(now);
        put(at_work, now);
    } while (now.left > 0);
    if constexpr (!SHARES) asm volatile("cp.async.wait_all;" ::: "memory");      // (blocks behind the last)
}

// The pieces of a head and tile of rows that several CTAs shared, in their order: a warp takes 32 elements of a row at a time, four groups
// of eight lanes every fourth piece.  How the blocks were shared out is found out while the kernel in front still runs.
constexpr int kJoinWarps = 4, kJoinAhead = 8;
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32)
cache_attention_join_kernel(AttArgs a, int NR, Divisor rows, int items, int most) {
    const int segs = a.H * (int)a.RT.d, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = lane % 8, by = lane / 8;
    int all = 0, longest = 0;
    for (int i = lane; i < a.B; i += 32) {
        const int v = blocks_of(a, i);
        all += v;
        longest = max(longest, v);
    }
    const int total = __reduce_add_sync(0xffffffffu, all) * segs;
    longest = __reduce_max_sync(0xffffffffu, longest);
    const Shares share = shares_of(total, longest, a.B * segs, most);
    if (share.whole) items = 0;
    bool waited = false;
    for (int item = blockIdx.x * kJoinWarps + warp; item < items; item += gridDim.x * kJoinWarps) {
        const int chunk = item % (D / 32), sr = item / (D / 32), s = quotient(sr, rows), rl = sr - s * (int)rows.d;
        const int b = s / segs, seg = s - b * segs, h = quotient(seg, a.RT), r = (seg - h * (int)a.RT.d) * NR + rl;
        if (r >= (int)a.R.d * a.Tq) continue;
        int before = 0;
        for (int i = lane; i < b; i += 32) before += blocks_of(a, i);
        before = __reduce_add_sync(0xffffffffu, before);
        const int blocks = blocks_of(a, b), from = before * segs + seg * blocks;
        const int c0 = blocks > 0 ? holder_of(share, from) : 0, n = blocks > 0 ? holder_of(share, from + blocks - 1) - c0 + 1 : 0;
        if (n == 1) continue;                              // one CTA had it all, and wrote the result
        if (!waited) grid_dependency_wait();
        waited = true;
        const size_t size = (size_t)NR * (D + 3);
        const auto slot = [&](int c) { return a.part + (size_t)(2 * (c0 + c) + (c == 0 ? 1 : 0)) * size; };
        float v[4] = {}, sum = 0.f, weight = 0.f, base = kNoLogit;
        for (int first = 0; first < n; first += 32) {
            const int m = min(n - first, 32);
            float4 x[kJoinAhead];
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i)
                if (by + 4 * i < m) x[i] = *reinterpret_cast<const float4*>(slot(first + by + 4 * i) + rl * D + chunk * 32 + 4 * col);
            float mine = kNoLogit, part = 0.f, mass = 0.f;
            if (lane < m) {
                const float* const p = slot(first + lane) + NR * D + rl;
                mine = p[0];
                part = p[NR];
                mass = p[2 * NR];
            }
            float top = fmaxf(mine, base);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float keep = ex2_approx(base - top), f = lane < m ? ex2_approx(mine - top) : 0.f;
            base = top;
            sum = fmaf(sum, keep, part * f);
            weight = fmaf(weight, keep, mass * f);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= keep;
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const float w = __shfl_sync(0xffffffffu, f, by + 4 * i);
                if (by + 4 * i < m) {
                    v[0] = fmaf(x[i].x, w, v[0]);
                    v[1] = fmaf(x[i].y, w, v[1]);
                    v[2] = fmaf(x[i].z, w, v[2]);
                    v[3] = fmaf(x[i].w, w, v[3]);
                }
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, off);
            weight += __shfl_xor_sync(0xffffffffu, weight, off);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] += __shfl_xor_sync(0xffffffffu, v[e], 8);
            v[e] += __shfl_xor_sync(0xffffffffu, v[e], 16);
        }
        const int tq = quotient(r, a.R), hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
        const bool none = sum == 0.f;                      // (no row seen, an empty sample's among them)
        const float inv = none ? 0.f : 1.f / weight;
        if (by == 0)
            *reinterpret_cast<uint2*>(a.io.out + b * a.io.ob + hq * a.io.oh + tq * a.io.ot + chunk * 32 + 4 * col) =
                make_uint2(bf16x2(v[0] * inv, v[1] * inv), bf16x2(v[2] * inv, v[3] * inv));
        if (a.lse && chunk == 0 && lane == 0) a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = none ? MINUS_INF : (base + __log2f(sum)) * kLn2;
    }
    if (!waited) grid_dependency_wait();                   // (what comes behind takes this kernel's end for that of the one in front)
}

struct Plan {
    int NT, RT, ctas;                                      // ctas: of the shares; 0: a CTA a head and tile of rows
    bool wide;                                             // such CTAs of eight warps
};

Plan plan_of(int B, int H, int Ncap, int d, int Tq, int Hq, int sms) {
    Plan p;
    const int64_t rows = (int64_t)(Hq / H) * Tq;
    // (tiles of 32 rows leave an SM eight warps: 32 rows of 16 heads, 16000 tokens 40.9 us, in tiles of 16 36.7)
    p.NT = rows <= 8 ? 1 : rows > 16 && rows <= 24 && d != 256 ? 3 : 2;
    // Few heads, and not too much to read for each tile again: tiles as narrow as leave an SM for each.  20 rows of 64 heads, 733 tokens: 9.0 us in
    // tiles of 16, 11.4 of 24; 64 rows of 16 heads, 1000 tokens: 9.5 in tiles of 8, 16.9 of 32; 20 rows of 8, 8000: 14.8 and 19.0 of 24; but
    // 20 rows of 32, 4000: 24.2 in tiles of 8, 23.3 of 24.
    for (int n = 1; n < p.NT; ++n) {
        const int64_t tiles = (int64_t)B * H * ((rows + 8 * n - 1) / (8 * n));
        if (tiles <= sms && tiles * (Ncap / kCacheBlock) <= 6400) {
            p.NT = n;
            break;
        }
    }
    p.RT = (int)((rows + 8 * p.NT - 1) / (8 * p.NT));
    const int slots = sms * ctas_per_sm(d, p.NT);
    const int64_t segs = (int64_t)B * H * p.RT, blocks = Ncap / kCacheBlock;
    p.ctas = 0;
    // The lengths are on the device; the plan takes all samples for as long as the cache has room, so that it is the same for every call of a
    // sequence that grows.  Blocks are shared out where that costs less (pieces, their join, the lengths in front) than what CTAs with a head
    // each leave idle, which is the SMs that have one head fewer than others.  Heads of 128, one query, all as long as the cache: 160 heads of
    // 2048 tokens 24.5 us and 23.0 shared out, of 4096 43.0 and 32.8; 288 of 4096 44.5 and 49.3; 384 of 1536 27.7 and 35.6, of 6144 92 and 85; 512 of
    // 4096 80.5 and 83.0; 2048 of 4096 256 and 281.  The other way round for few heads: 8 of 1056 10.0 and 9.2, 64 of 1536 12.1 and 11.9, 128 of
    // 4096 27.5 and 29.1.  Batches of which most samples are far shorter are better off with a CTA a head (512, a quarter of 4096 on
    // average, up to all: 35.2 us and 61.6), those between a quarter and all the other way (60.9 and 56.0).
    // (Up to four rounds of heads: what launch() has room for.)
    const bool one = segs <= sms, two = !one && segs <= 2 * sms && d * p.NT <= 128;
    bool whole = blocks <= kWholeBlocks || segs >= 4 * slots || segs * blocks >= 0x7fff0000;
    if (!whole && one) whole = blocks <= 128 && blocks * (27 * sms - 25 * segs) <= 675 * sms;
    if (!whole && !one) whole = blocks * ((segs + sms - 1) / sms * sms - segs) <= (40 + 30 * p.NT) * sms;
    // Eight warps where a head has an SM, or half of one.  64 heads of 512 tokens: 7.1 us with four, 6.5 with eight, of 2048 19.5 and 14.9; 160 of
    // 640 10.1 and 10.4, of 800 12.4 and 12.2, of 2048 26.0 and 24.5; 288 of 640 10.6 and 11.0, of 1536 21.4 and 21.4, of 4096 47.9 and 44.5.
    p.wide = whole && (one ? blocks > kWarps : two && blocks > kWholeBlocks);
    if (!whole) p.ctas = slots;
    return p;
}

size_t part_bytes(const Plan& p, int d) { return align_up((size_t)2 * p.ctas * 8 * p.NT * (d + 3) * sizeof(float), 256); }

template <int D, int NT, int W>
constexpr size_t smem_of() {
    return (size_t)W * kStages * CacheBlock<D>::kBytes + W * 2048 + 3 * W * 8 * NT * 4 + NT * 32 * sizeof(QueryOperand<D / 32>) +
           kStages * NT * (D / 32) * 512 + W * 2 * sizeof(Walk) + 4;
}
template <int D, int NT>
int launch(AttArgs a, const Plan& p, cudaStream_t stream) {
    static DoneOnDevice done[3];
    const bool shares = p.ctas > 0;
    const size_t smem = shares ? smem_of<D, NT, kWarps>() + (size_t)(2 * a.B + 2) * 4 : p.wide ? smem_of<D, NT, 8>() : smem_of<D, NT, kWarps>();
    const auto kern = shares ? cache_attention_kernel<D, NT, true, kWarps> : p.wide ? cache_attention_kernel<D, NT, false, 8> : cache_attention_kernel<D, NT, false, kWarps>;
    int rc = allow_dynamic_smem(kern, (p.wide ? smem_of<D, NT, 8>() : smem_of<D, NT, kWarps>()) + (shares ? 20480 : 0), done[shares ? 1 : p.wide ? 2 : 0]);
    if (rc != VITCOP_OK) return rc;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(shares ? p.ctas : a.B * a.H * p.RT));
    cfg.blockDim = dim3((p.wide ? 8 : kWarps) * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    {
        KernelTimeScope timed("cache_attention_kernel", stream);
        rc = record_cuda(cudaLaunchKernelEx(&cfg, kern, a));
        if (rc != VITCOP_OK || !shares) return rc;
    }
    const int rows = (int)a.R.d * a.Tq < 8 * NT ? (int)a.R.d * a.Tq : 8 * NT;      // that a tile has at most
    const int64_t items = (int64_t)a.B * a.H * a.RT.d * rows * (D / 32);
    const int64_t wave = sm_count() * 8, ctas = (items + kJoinWarps - 1) / kJoinWarps;
    cfg.gridDim = dim3((unsigned)(ctas < wave ? ctas : wave));
    cfg.blockDim = dim3(kJoinWarps * 32);
    cfg.dynamicSmemBytes = 0;
    KernelTimeScope timed("cache_attention_join_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, cache_attention_join_kernel<D>, a, 8 * NT, divisor(rows), (int)items, p.ctas));
}

}  // namespace

int sm_count() {
    static std::atomic<int> known[kMaxDevices];
    std::atomic<int>& k = known[current_device()];
    int v = k.load(std::memory_order_relaxed);
    if (v == 0) {
        if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, current_device()) != cudaSuccess || v <= 0) v = 148;
        k.store(v, std::memory_order_relaxed);
    }
    return v;
}

size_t cache_attention_workspace_bytes(int B, int H, int Ncap, int d, int Tq, int Hq) {
    if (B < 1 || H < 1 || Hq < 1 || Tq < 1) return kStatusBytes;
    if (rows_kernel_takes(B, H, Ncap, (int64_t)Hq / H * Tq, d)) return rows_workspace_bytes(B, H, Ncap, d, Tq, Hq);
    const Plan p = plan_of(B, H, Ncap, d, Tq, Hq, sm_count());
    return kStatusBytes + part_bytes(p, d);
}

int launch_cache_attention(const CacheQueries& io, const void* cache, int B, int Hq, int H, int Tq, int d, int Ncap,
                           const int32_t* cache_len, float scale, bool causal, float* lse, void* workspace, cudaStream_t stream) {
    const bool many = rows_kernel_takes(B, H, Ncap, (int64_t)Hq / H * Tq, d);
    const Plan p = plan_of(B, H, Ncap, d, Tq, Hq, sm_count());
    if ((int64_t)B * H * p.RT > 0x7fffffff || (int64_t)Hq / H * Tq > 0x7fffffff - 64) return VITCOP_ERR_UNSUPPORTED;
    AttArgs a;
    a.io = io;
    a.cache = static_cast<const uint8_t*>(cache);
    a.cache_len = cache_len;
    a.lse = lse;
    a.status = static_cast<int*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kStatusBytes);
    a.B = B; a.Hq = Hq; a.H = H; a.R = divisor(Hq / H); a.Tq = Tq; a.Ncap = Ncap; a.RT = divisor(p.RT); a.causal = causal ? 1 : 0;
    a.sign = scale < 0.f ? 0x80008000u : 0u;
    // (0 would make NaN of the -inf of tokens that are not seen; the smallest number above it leaves no logit of fp32 more than 2^-21)
    a.scale_log2 = fmaxf(fabsf(scale) * kLog2e, 0x1p-149f);
    if (many) return launch_cache_attention_rows(a, d, workspace, stream);
    if (d == 64) return p.NT == 1 ? launch<64, 1>(a, p, stream) : p.NT == 2 ? launch<64, 2>(a, p, stream) : launch<64, 3>(a, p, stream);
    if (d == 128) return p.NT == 1 ? launch<128, 1>(a, p, stream) : p.NT == 2 ? launch<128, 2>(a, p, stream) : launch<128, 3>(a, p, stream);
    return p.NT == 1 ? launch<256, 1>(a, p, stream) : launch<256, 2>(a, p, stream);
}

}  // namespace vitcop
