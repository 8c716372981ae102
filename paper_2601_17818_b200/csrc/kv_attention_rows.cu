// Attention over the cache in 4 bits for many query rows (a question, a chunk of a prompt): 128 rows of a head a CTA, tcgen05.
//
// Tokens come in tiles of 64.  Eight warps turn a tile into operands: codes of K as the bf16 c - 8, exactly, codes of V as the values
// they stand for, transposed, in fp16 (three bits more than bf16 has) times a power of two that the largest scale and centre so far
// allow.  With G = d / 32 groups of a row the logits are
//     z = sum over g of s_g (q_g . (c - 8)_g)  +  sum over g of m_g sum(q_g)
// G products of their own (q as it is, bf16), whose fp32 sums the scales multiply behind tensor memory, and one more for the centres with
// sum(q_g) split into three bf16.  Eight warps, two threads a row (32 tokens each), make the weights of the logits and write them back as
// operand of the second product, which stays in tensor memory; a row's maximum is moved only when a logit has passed it by 2^8.
// (Weights in fp16 too, 2^-7 .. 2^15 at the top: the smallest that count are 2^-31 of the largest.)
// Every operand is rows of 128 bytes in the 128-byte swizzle.  Waits are bounded: a CTA that gives up reports it, and the join,
// which always follows, sets the status word.
// Bound by the instructions of unpacking and softmax: 2700 cycles a tile, 57 % of the issue slots.  4 x 4 heads of 128, 448 rows, 1280
// tokens: 30 us with the join, 155 TFLOP/s, of which start and end are 10; 512 rows of 32 heads, 4000 tokens: 104 us, 320 TFLOP/s.
#include <cuda_fp16.h>

#include "gram.cuh"
#include "kv_attention.cuh"
#include "tcgen05.cuh"

namespace vitcop {
namespace {

constexpr int kRows = 128, kTokens = 64;
constexpr int kSoftmaxThreads = 256, kUnpackThreads = 256, kThreads = kSoftmaxThreads + kUnpackThreads + 64;
constexpr int kStages = 3, kMostSplits = 16;
constexpr uint32_t kTmem = 512;
enum { kRoleUnpack = 1, kRoleMma = 2, kRoleSoftmax = 4 };
// What a CTA reports: whether a wait ran out, and a bit for each of its rows that fp16 does not hold, which the join does anew in fp32.
// Weights are off by 2^-25 at most where they are small, and values of V (in the units that their power of two makes: the largest is below 2^15)
// by 2^-25, so that a row's sum over the N tokens of the CTA is off by N 2^-25 V + W 2^-25 in a group of 32 elements whose largest value is
// V, with W the sum of the row's weights, 2^7 at least.  A row is reported where that is more than 2^-8 of the largest of the group's 32
// sums: it looks at little but tokens with far smaller values than others have, or the whole group is some 2^-25 of another.
struct Report {
    uint32_t gave_up, rows[kRows / 32];
};
constexpr float kLostOf = 0x1p-17f;                        // 2^-25 over 2^-8

template <int D>
struct RowsSmem {
    static constexpr int kSubs = D / 64;
    static constexpr int kQ = 0;                                       // [D / 64][128 rows][128 bytes]
    static constexpr int kSums = kQ + kSubs * 16384;                   // [128 rows][128 bytes], 32 of which are used
    static constexpr int kP = kSums + 16384;                           // [128 rows][64 tokens]
    static constexpr int kStage = kP + 16384;                          // kStages of them:
    static constexpr int kK = 0;                                       //   [D / 64][64 tokens][128 bytes]
    static constexpr int kV = kK + kSubs * 8192;                       //   [D elements, and 16 rows: ones and zeros][64 tokens]
    static constexpr int kC = kV + (D + 16) * 128;                            //   [64 tokens][128 bytes]
    static constexpr int kS = kC + 8192;                               //   fp32 [G][64 tokens]
    static constexpr int kStageBytes = kS + 1024;
    static constexpr int kRaw = kStage + kStages * kStageBytes;              // two tiles as they lie in the cache
    static constexpr int kRawBytes = 2 * CacheBlock<D>::kBytes;
    static constexpr int kBars = kRaw + 2 * kRawBytes;
    // What the two threads of a row tell each other, fp32 [2][128 rows] each: maxima, tile by tile, and the sums at the end.  (Arrays of their
    // own: nothing holds a thread up between its partner's last maximum and its own sum.)
    static constexpr int kPairs = kBars + 256;
    static constexpr int kEnds = kPairs + 1024;
    static constexpr int kTable = kEnds + 1024;                       // fp16 [2][G][64 tokens]: scales and centres of V, times the power of two
    static constexpr int kAnew = kTable + 1024;                        // [2][4] rows to be done anew, as the two halves of the softmax warps find
    static constexpr int kBytes = kAnew + 32 + 1024;                     // (and what aligning to 1024 takes)
};

struct RowsArgs {
    AttArgs a;
    Report* reports;                                       // one a CTA
    int splits;
    unsigned long long wait_ns;
    int expire_roles;
    __device__ __forceinline__ unsigned long long limit_of(int role) const { return (expire_roles & role) ? 0ull : wait_ns; }
};

// Byte of 16-byte piece c of row r.
__device__ __forceinline__ int at_swizzled(int r, int c) { return r * 128 + ((c ^ (r & 7)) << 4); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void unpack_bar() { asm volatile("bar.sync 2, 256;" ::: "memory"); }
__device__ __forceinline__ bool unpack_bar_or(bool pred) {     // the same answer for all of them
    uint32_t out;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, 2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(out) : "r"((uint32_t)pred) : "memory");
    return out != 0;
}

// As tc_mma_bf16 and tc_commit, called by a warp of which one lane issues.
__device__ __forceinline__ void mma_elected(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_elected(uint32_t bar) {
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int N>
__device__ __forceinline__ void words(uint32_t (&w)[N], const uint8_t* p) {
    if constexpr (N == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

template <int N>
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[N][8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int n = 0; n < N; ++n)                            // (no use of the registers in front of the wait)
        asm volatile("" : "+r"(r[n][0]), "+r"(r[n][1]), "+r"(r[n][2]), "+r"(r[n][3]), "+r"(r[n][4]), "+r"(r[n][5]), "+r"(r[n][6]), "+r"(r[n][7]));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32]) {
    const auto u = [&](int i) { return __float_as_uint(v[i]); };
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(u(0)), "r"(u(1)), "r"(u(2)), "r"(u(3)), "r"(u(4)), "r"(u(5)), "r"(u(6)), "r"(u(7)), "r"(u(8)), "r"(u(9)), "r"(u(10)),
        "r"(u(11)), "r"(u(12)), "r"(u(13)), "r"(u(14)), "r"(u(15)), "r"(u(16)), "r"(u(17)), "r"(u(18)), "r"(u(19)), "r"(u(20)), "r"(u(21)),
        "r"(u(22)), "r"(u(23)), "r"(u(24)), "r"(u(25)), "r"(u(26)), "r"(u(27)), "r"(u(28)), "r"(u(29)), "r"(u(30)), "r"(u(31))
        : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(__float_as_uint(v)) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
cache_attention_rows_kernel(RowsArgs k) {
    using L = CacheBlock<D>;
    using S = RowsSmem<D>;
    constexpr int G = L::G;
    const AttArgs& a = k.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const uint32_t bar_full = base + S::kBars, bar_empty = bar_full + 8 * kStages, bar_s = bar_empty + 8 * kStages, bar_read = bar_s + 8, bar_p = bar_s + 16,
                   bar_pv = bar_s + 24, bar_drain = bar_s + 32, bar_q = bar_s + 48;     // (two drains)
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + S::kBars + 128);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + S::kBars + 132);
    int* const moved = reinterpret_cast<int*>(smem + S::kBars + 160);          // [3] a row's maximum has to move, tile by tile
    uint32_t* const bounds = reinterpret_cast<uint32_t*>(smem + S::kBars + 192);     // [8] largest value of V that a warp has found possible
    int* const exponents = reinterpret_cast<int*>(smem + S::kBars + 224);           // [kStages] of that power of two, as a float's bits have it
    float* const pairs = reinterpret_cast<float*>(smem + S::kPairs);
    float* const ends = reinterpret_cast<float*>(smem + S::kEnds);
    uint32_t* const greatest = reinterpret_cast<uint32_t*>(smem + S::kBars + 176);   // [G] largest value of V that a group has, as a float's bits
    uint32_t* const anew = reinterpret_cast<uint32_t*>(smem + S::kAnew);
    int* const first_bad = reinterpret_cast<int*>(smem + S::kBars + 144);       // [G] first token whose values of V are no numbers
    const int tid = threadIdx.x, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(bar_full + 8 * i, kUnpackThreads);
            mbar_init(bar_empty + 8 * i, 1);
        }
        mbar_init(bar_s, 1);
        mbar_init(bar_read, kSoftmaxThreads);
        mbar_init(bar_p, kSoftmaxThreads);
        mbar_init(bar_pv, 1);
        mbar_init(bar_drain, 1);
        mbar_init(bar_drain + 8, 1);
        mbar_init(bar_q, kRows);
        *abort_flag = 0;
        moved[0] = moved[1] = moved[2] = 0;
        for (int i = 0; i < G; ++i) {
            first_bad[i] = 0x7fffffff;
            greatest[i] = 0;
        }
        for (int i = 0; i < 8; ++i) anew[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // the row of ones, whose product is the sum of the weights as they are rounded: what the output is divided by.  (In front of
    // the barrier: where there is no tile, the output goes through the same bytes with no other in between.)
    if (tid >= kSoftmaxThreads && tid < kSoftmaxThreads + kUnpackThreads)
        for (int i = tid - kSoftmaxThreads; i < kStages * 128; i += kUnpackThreads)
            *reinterpret_cast<uint4*>(smem + S::kStage + (i >> 7) * S::kStageBytes + S::kV + D * 128 + (i & 127) * 16) =
                (i & 127) < 8 ? make_uint4(0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u) : make_uint4(0, 0, 0, 0);
    if (warp == kThreads / 32 - 1) tmem_alloc(smem_u32(tmem_slot), kTmem);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0), tmem_z = tmem, tmem_c = tmem + 4 * kTokens, tmem_o = tmem_c + kTokens;
    grid_dependency_wait();
    grid_dependency_launch_dependents();                   // (the join's CTAs, which wait for this grid to end)

    const int split = blockIdx.x % k.splits, seg = blockIdx.x / k.splits, segs = a.H * (int)a.RT.d, b = seg / segs, hs = seg - b * segs;
    const int h = quotient(hs, a.RT), row0 = (hs - h * (int)a.RT.d) * kRows, rows = (int)a.R.d * a.Tq;
    const int len = a.cache_len ? max(0, min(__ldcg(a.cache_len + b), a.Ncap)) : a.Ncap;
    const int last = min(row0 + kRows, rows) - 1;
    const int most = a.causal ? max(0, len - a.Tq + quotient(last, a.R) + 1) : len;
    const int least = a.causal ? max(0, len - a.Tq + quotient(row0, a.R) + 1) : len;
    const int tiles = (most + kTokens - 1) / kTokens;
    const int each = tiles / k.splits, more = tiles - each * k.splits, t0 = split * each + min(split, more), n = each + (split < more ? 1 : 0);
    const uint8_t* const head = a.cache + ((int64_t)b * a.H + h) * (a.Ncap / kCacheBlock) * L::kBytes;

    // this thread's row as operand
    const int rl = tid & (kRows - 1), r = row0 + rl, tq = r < rows ? quotient(r, a.R) : 0, hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
    int limit = 0;
    if (tid < kSoftmaxThreads) limit = r < rows ? (a.causal ? max(0, len - a.Tq + tq + 1) : len) : 0;
    if (tid < kRows) {
        const bool there = r < rows;
        const __nv_bfloat16* const src = a.io.q + (there ? b * a.io.qb + hq * a.io.qh + tq * a.io.qt : 0);
        float total[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            float x = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint4 v = there ? __ldcg(reinterpret_cast<const uint4*>(src + i * 32 + c * 8)) : make_uint4(0, 0, 0, 0);
                v = make_uint4(v.x ^ a.sign, v.y ^ a.sign, v.z ^ a.sign, v.w ^ a.sign);
                x += ((bf16lo(v.x) + bf16hi(v.x)) + (bf16lo(v.y) + bf16hi(v.y))) + ((bf16lo(v.z) + bf16hi(v.z)) + (bf16lo(v.w) + bf16hi(v.w)));
                // elements 0 and 4, 1 and 5, 2 and 6, 3 and 7, as the codes lie
                *reinterpret_cast<uint4*>(smem + S::kQ + (i / 2) * 16384 + at_swizzled(tid, (i & 1) * 4 + c)) =
                    make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
            }
            total[i] = x;
        }
        // part p of group i is element p G + i of the product with the centres
        float part[16] = {};
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const float first = __bfloat162float(__float2bfloat16_rn(total[i])), second = __bfloat162float(__float2bfloat16_rn(total[i] - first));
            part[i] = first;
            part[G + i] = second;
            part[2 * G + i] = (total[i] - first) - second;
        }
        *reinterpret_cast<uint4*>(smem + S::kSums + at_swizzled(tid, 0)) =
            make_uint4(bf16x2(part[0], part[1]), bf16x2(part[2], part[3]), bf16x2(part[4], part[5]), bf16x2(part[6], part[7]));
        *reinterpret_cast<uint4*>(smem + S::kSums + at_swizzled(tid, 1)) =
            make_uint4(bf16x2(part[8], part[9]), bf16x2(part[10], part[11]), bf16x2(part[12], part[13]), bf16x2(part[14], part[15]));
        fence_async_proxy();
        mbar_arrive(bar_q);
    }

    if (tid < kSoftmaxThreads) {
        // ------------------------------------------------------------------ softmax: two threads a row, 32 tokens each
        const unsigned long long lim = k.limit_of(kRoleSoftmax);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        constexpr int kHalf = kTokens / 2;
        const int half = warp >> 2;
        float top = kNoLogit, sum = 0.f;                   // in powers of two; weights are 2^(logit - top)
        int exponent = 0;                                  // of V, as the sums have it
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int token0 = (t0 + i) * kTokens + half * kHalf;
            const float* const scale = reinterpret_cast<const float*>(smem + S::kStage + i % kStages * S::kStageBytes + S::kS) + half * kHalf;
            ok = __all_sync(0xffffffffu, mbar_wait(bar_s, i & 1, abort_flag, lim));
            tc_fence_after();
            float z[kHalf];
#pragma unroll
            for (int c = 0; c < kHalf / 8; ++c) {
                uint32_t x[G + 1][8];
                tmem_ld8_issue(tmem_c + lanes + half * kHalf + 8 * c, x[G]);
#pragma unroll
                for (int g = 0; g < G; ++g) tmem_ld8_issue(tmem_z + lanes + g * kTokens + half * kHalf + 8 * c, x[g]);
                tmem_wait_ld(x);
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    f32x2 lo = pack2(__uint_as_float(x[G][e]), __uint_as_float(x[G][e + 1])), hi = pack2(__uint_as_float(x[G][e + 2]), __uint_as_float(x[G][e + 3]));
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float4 f = *reinterpret_cast<const float4*>(scale + g * kTokens + 8 * c + e);
                        lo = fma2(pack2(__uint_as_float(x[g][e]), __uint_as_float(x[g][e + 1])), pack2(f.x, f.y), lo);
                        hi = fma2(pack2(__uint_as_float(x[g][e + 2]), __uint_as_float(x[g][e + 3])), pack2(f.z, f.w), hi);
                    }
                    const float2 u = unpack2(lo), v = unpack2(hi);
                    z[8 * c + e] = u.x;
                    z[8 * c + e + 1] = u.y;
                    z[8 * c + e + 2] = v.x;
                    z[8 * c + e + 3] = v.y;
                }
            }
            tc_fence_before();
            mbar_arrive(bar_read);
            if (token0 + kHalf > least) {
                const int seen = limit - token0;
#pragma unroll
                for (int e = 0; e < kHalf; ++e)
                    if (e >= seen) z[e] = MINUS_INF;
            }
            float high = z[0];
#pragma unroll
            for (int e = 1; e < kHalf; ++e) high = fmaxf(high, z[e]);
            high *= a.scale_log2;
            if (high - top > 15.f) moved[i % 3] = 1;
            if (tid == 0) moved[(i + 1) % 3] = 0;          // (read last two barriers ago)
            // the product behind has read the weights, and its sums stand still (one warp asks, the others have the barrier)
            if (i > 0 && warp == 0) ok = mbar_wait(bar_pv, (i - 1) & 1, abort_flag, lim) && ok;
            if (epi_bar_or<kSoftmaxThreads>(!ok)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const int next = exponents[i % kStages];
            if (moved[i % 3] || (next != exponent && i > 0)) {         // (the same for all)
                pairs[half * kRows + rl] = high;
                epi_bar_sync<kSoftmaxThreads>();
                const float now = fmaxf(top, fmaxf(high, pairs[(half ^ 1) * kRows + rl]) - 7.f), keep = ex2_approx(top - now);
                const float less = keep * __int_as_float(max(0, 127 + exponent - next) << 23);
                top = now;
                sum *= keep;
                if (i > 0) {
#pragma unroll 1
                    for (int c = half * (G / 2); c < (half + 1) * (G / 2); ++c) {
                        float v[32];
                        tmem_ld32(tmem_o + lanes + 32 * c, v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] *= less;
                        tmem_st32(tmem_o + lanes + 32 * c, v);
                    }
                    if (half == 0) {
                        uint32_t w[1][8];
                        tmem_ld8_issue(tmem_o + lanes + D, w[0]);
                        tmem_wait_ld(w);
                        tmem_st1(tmem_o + lanes + D, __uint_as_float(w[0][0]) * keep);
                    }
                }
            }
            exponent = next;
            float more = 0.f;
#pragma unroll
            for (int c = 0; c < kHalf / 8; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p0 = ex2_approx(fmaf(z[8 * c + 2 * e], a.scale_log2, -top)), p1 = ex2_approx(fmaf(z[8 * c + 2 * e + 1], a.scale_log2, -top));
                    if (e & 1) more += p0 + p1; else sum += p0 + p1;
                    w[e] = f16x2(p0, p1);
                }
                *reinterpret_cast<uint4*>(smem + S::kP + at_swizzled(rl, half * 4 + c)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            sum += more;
            fence_async_proxy();
            tc_fence_before();
            mbar_arrive(bar_p);
        }
        if (ok && n > 0 && warp == 0) ok = mbar_wait(bar_pv, (n - 1) & 1, abort_flag, lim);
        ends[half * kRows + rl] = sum;
        if (!epi_bar_or<kSoftmaxThreads>(!ok)) {
            tc_fence_after();
            sum += ends[(half ^ 1) * kRows + rl];
            const bool none = sum == 0.f, alone = k.splits == 1;
            uint32_t weight[1][8] = {};
            if (n > 0) {
                tmem_ld8_issue(tmem_o + lanes + D, weight[0]);
                tmem_wait_ld(weight);
            }
            const float total = __uint_as_float(weight[0][0]), inv = none ? 0.f : __int_as_float((exponent - 14) << 23) / total;
            const float lost_weights = (float)(n * kTokens) * kLostOf * __int_as_float((268 - exponent) << 23), lost_values = total * kLostOf;
            bool redo = false;
            float* const part = a.part + (size_t)blockIdx.x * kRows * (D + 3);
            // (32 rows by 32 elements a warp, turned in shared memory that the tiles have left: 8 lanes then write a row)
            float* const turn = reinterpret_cast<float*>(smem + S::kStage) + warp * 32 * 36;
            const int lane = tid & 31;
#pragma unroll 1
            for (int c = half * (G / 2); c < (half + 1) * (G / 2); ++c) {
                float v[32];
                if (n > 0) {
                    tmem_ld32(tmem_o + lanes + 32 * c, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0.f;
                }
                // (all of a group may be 0, and the sums then are)
                const float most_value = __uint_as_float(greatest[c]);
                float largest = 0.f;
#pragma unroll
                for (int e = 0; e < 32; ++e) largest = fmaxf(largest, fabsf(v[e]));
                redo |= most_value > 0.f && largest < fmaf(most_value, lost_weights, lost_values);
                const bool bad = first_bad[c] < limit;     // a row of V that is no number, and that this query sees
                const float times = bad ? __int_as_float(0x7fc00000) : inv;
#pragma unroll
                for (int g = 0; g < 8; ++g)                // (column 8 i + g of a group is its element 4 g + i)
                    *reinterpret_cast<float4*>(turn + lane * 36 + 4 * g) = make_float4(v[g] * times, v[8 + g] * times, v[16 + g] * times, v[24 + g] * times);
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int row = (warp & 3) * 32 + 4 * j + (lane >> 3), q = row0 + row;
                    const float4 o = *reinterpret_cast<const float4*>(turn + (4 * j + (lane >> 3)) * 36 + 4 * (lane & 7));
                    if (q >= rows) continue;
                    if (alone) {
                        const int qt = quotient(q, a.R), qh = h * (int)a.R.d + (q - qt * (int)a.R.d);
                        *reinterpret_cast<uint2*>(a.io.out + b * a.io.ob + qh * a.io.oh + qt * a.io.ot + c * 32 + 4 * (lane & 7)) =
                            make_uint2(bf16x2(o.x, o.y), bf16x2(o.z, o.w));
                    } else {
                        *reinterpret_cast<float4*>(part + row * D + c * 32 + 4 * (lane & 7)) = o;
                    }
                }
                __syncwarp();
            }
            const uint32_t which = __ballot_sync(0xffffffffu, redo && r < rows && !none);
            if (lane == 0) anew[warp] = which;
            if (r < rows && half == 0) {
                if (!alone) {
                    part[kRows * D + rl] = top;
                    part[kRows * D + kRows + rl] = sum;
                    part[kRows * D + 2 * kRows + rl] = __uint_as_float(weight[0][0]);
                } else if (a.lse) {
                    a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = none ? MINUS_INF : (top + __log2f(sum)) * kLn2;
                }
            }
        }
    } else if (tid < kSoftmaxThreads + kUnpackThreads) {
        // ------------------------------------------------------------------ unpack
        const unsigned long long lim = k.limit_of(kRoleUnpack);
        const int u = tid - kSoftmaxThreads, blocks = (len + kCacheBlock - 1) / kCacheBlock;
        const auto fetch = [&](int i) {                    // (a tile's second block may be behind the last there is)
            if (i < n) {
                const int first = (t0 + i) * 2, pieces = min(2, blocks - first) * (L::kBytes / 16);
                const uint8_t* const src = head + (int64_t)first * L::kBytes;
                const uint32_t dst = base + S::kRaw + (i & 1) * S::kRawBytes;
                for (int c = u; c < pieces; c += kUnpackThreads)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 16 * c), "l"(src + 16 * c) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        fetch(0);
        fetch(1);
        uint16_t* const table = reinterpret_cast<uint16_t*>(smem + S::kTable);
        int exponent = 16;
        uint32_t mine = 0;                                 // largest value of V in this thread's group, in its tokens
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            if (i >= kStages && u < 32) ok = mbar_wait(bar_empty + 8 * (i % kStages), (i / kStages - 1) & 1, abort_flag, lim);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            if (unpack_bar_or(!ok || *abort_flag)) break;
            const uint8_t* const raw = smem + S::kRaw + (i & 1) * S::kRawBytes;
            uint8_t* const stage = smem + S::kStage + i % kStages * S::kStageBytes;
            const int token0 = (t0 + i) * kTokens;
            // V's scale and centre of a token and group, a thread each, and the largest value that they allow.  What is no number would
            // reach rows that do not see it: it is a zero here, and those that do see it are told.  So are tokens that no row sees.
            float scale = 0.f, centre = 0.f;
            if (u < kTokens * G) {
                const int token = u / G, g = u % G, rb = token & 31;
                const uint8_t* const block = raw + (token >> 5) * L::kBytes;
                const float f = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(block + L::kVScale + (rb * G + g) * 2) << 16);
                const float m = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(block + L::kVCentre + (g * 32 + rb) * 2) << 16);
                if (token0 + token < most) {
                    if (f == f) {
                        scale = f;
                        centre = m;
                    } else {
                        atomicMin(first_bad + g, token0 + token);
                    }
                }
            }
            const uint32_t here = __float_as_uint(fmaf(8.f, fabsf(scale), fabsf(centre))), most_here = __reduce_max_sync(0xffffffffu, here);
            mine = max(mine, here);
            if ((u & 31) == 0) bounds[u >> 5] = most_here;
            {   // K: a thread a quarter of a token's row
                const int row = u >> 2, t = u & 3, rb = row & 31;
                const uint8_t* const block = raw + (row >> 5) * L::kBytes;
                uint32_t w[G];
                words<G>(w, block + L::kKCodes + rb * (D / 2) + t * 4 * G);
#pragma unroll
                for (int g = 0; g < G; ++g)
                    *reinterpret_cast<uint4*>(stage + S::kK + (g / 2) * 8192 + at_swizzled(row, (g & 1) * 4 + t)) =
                        make_uint4(centred(code_pair(w[g])), centred(code_pair(w[g] >> 4)), centred(code_pair(w[g] >> 8)), centred(code_pair(w[g] >> 12)));
            }
            if (u < kTokens) {                             // centres three times over, scales
                const uint8_t* const block = raw + (u >> 5) * L::kBytes;
                const int rb = u & 31;
                uint32_t m[G / 2], s[G / 2];
                words<G / 2>(m, block + L::kKCentre + rb * 2 * G);
                words<G / 2>(s, block + L::kKScale + rb * 2 * G);
                *reinterpret_cast<uint4*>(stage + S::kC + at_swizzled(u, 0)) = G == 4 ? make_uint4(m[0], m[G / 2 - 1], m[0], m[G / 2 - 1]) : make_uint4(m[0], m[0], m[0], 0u);
                *reinterpret_cast<uint4*>(stage + S::kC + at_swizzled(u, 1)) = G == 4 ? make_uint4(m[0], m[G / 2 - 1], 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);
                float* const f = reinterpret_cast<float*>(stage + S::kS) + u;
#pragma unroll
                for (int g = 0; g < G; ++g) f[g * kTokens] = g & 1 ? bf16hi(s[g / 2]) : bf16lo(s[g / 2]);
            }
            unpack_bar();
            uint32_t bound = 0;
#pragma unroll
            for (int w = 0; w < kUnpackThreads / 32; ++w) bound = max(bound, bounds[w]);
            exponent = max(exponent, (int)(bound >> 23));  // (values times 2^(141 - exponent) are below 2^15)
            const float up = __int_as_float((268 - exponent) << 23);
            if (u < kTokens * G) {
                table[(u % G) * kTokens + u / G] = __half_as_ushort(__float2half_rn(scale * up));
                table[(G + u % G) * kTokens + u / G] = __half_as_ushort(__float2half_rn(centre * up));
            }
            if (u == 0) exponents[i % kStages] = exponent;
            unpack_bar();
            {   // V: a thread four elements of each group of two tokens
                const int g8 = u & 7, pair = u >> 3, rb = 2 * (pair & 15);
                const uint8_t* const block = raw + (pair >> 4) * L::kBytes;
                uint32_t x0[G / 2], x1[G / 2];
                words<G / 2>(x0, block + L::kVCodes + rb * (D / 2) + g8 * 2 * G);
                words<G / 2>(x1, block + L::kVCodes + (rb + 1) * (D / 2) + g8 * 2 * G);
                uint8_t* const to = stage + S::kV + at_swizzled(g8, pair >> 2) + (pair & 3) * 4;     // (rows 8 apart are 1024 bytes apart)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t x = __byte_perm(x0[g / 2], x1[g / 2], g & 1 ? 0x7632u : 0x5410u);
                    const uint32_t f = *reinterpret_cast<const uint32_t*>(table + g * kTokens + 2 * pair), m = *reinterpret_cast<const uint32_t*>(table + (G + g) * kTokens + 2 * pair);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {          // (1024 + c) - 1032 = c - 8
                        uint32_t y;
                        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(x >> (4 * e)), "r"(0x000F000Fu), "r"(0x64006400u));
                        asm("add.rn.f16x2 %0, %0, %1;" : "+r"(y) : "r"(0xE408E408u));
                        asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(y) : "r"(f), "r"(m));
                        *reinterpret_cast<uint32_t*>(to + (g * 4 + e) * 1024) = y;
                    }
                }
            }
            if (i == n - 1) {                              // (thread u has group u % G in all tiles; where G = 2 half of them have none)
#pragma unroll
                for (int off = G; off < 32; off <<= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, off));
                if ((u & 31) < G) atomicMax(greatest + (u & 31), mine);
            }
            fence_async_proxy();
            mbar_arrive(bar_full + 8 * (i % kStages));
            unpack_bar();                                  // (the raw tile has been read)
            fetch(i + 2);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp == kThreads / 32 - 2) {
        // ------------------------------------------------------------------ products with the queries
        // (the whole warp walks, so that the operands' addresses are known to be the same in all lanes; one lane issues)
        const unsigned long long lim = k.limit_of(kRoleMma);
        constexpr uint32_t idesc = umma_idesc_bf16(kRows, kTokens);
        int at = 0, phase = 0;
        const bool there = n > 0 && __all_sync(0xffffffffu, mbar_wait(bar_q, 0, abort_flag, lim));
        for (int i = 0; there && i < n; ++i) {
            const bool ok = mbar_wait(bar_full + 8 * at, phase, abort_flag, lim) && (i == 0 || mbar_wait(bar_read, (i - 1) & 1, abort_flag, lim));
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const uint32_t stage = base + S::kStage + at * S::kStageBytes;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint64_t dq = umma_desc_k128(base + S::kQ + (g / 2) * 16384) + (uint64_t)((g & 1) * 4);
                const uint64_t dk = umma_desc_k128(stage + S::kK + (g / 2) * 8192) + (uint64_t)((g & 1) * 4);
                mma_elected(tmem_z + g * kTokens, dq, dk, idesc, 0);
                mma_elected(tmem_z + g * kTokens, dq + 2, dk + 2, idesc, 1);
            }
            mma_elected(tmem_c, umma_desc_k128(base + S::kSums), umma_desc_k128(stage + S::kC), idesc, 0);
            commit_elected(bar_s);
            if (++at == kStages) {
                at = 0;
                phase ^= 1;
            }
        }
        commit_elected(bar_drain);                         // (waited for below)
    } else {
        // ------------------------------------------------------------------ products with the weights
        const unsigned long long lim = k.limit_of(kRoleMma);
        constexpr uint32_t idesc = umma_idesc_bf16(kRows, D + 16) & ~(1u << 7 | 1u << 10);       // (both operands fp16)
        int at = 0;
        for (int i = 0; i < n; ++i) {
            if (!__all_sync(0xffffffffu, mbar_wait(bar_p, i & 1, abort_flag, lim))) break;
            tc_fence_after();
            const uint64_t dp = umma_desc_k128(base + S::kP), dv = umma_desc_k128(base + S::kStage + at * S::kStageBytes + S::kV);
#pragma unroll
            for (int e = 0; e < kTokens / 16; ++e) mma_elected(tmem_o, dp + 2 * e, dv + 2 * e, idesc, i > 0 || e > 0 ? 1u : 0u);
            commit_elected(bar_pv);
            commit_elected(bar_empty + 8 * at);
            if (++at == kStages) at = 0;
        }
        commit_elected(bar_drain + 8);
    }
    __syncthreads();
    // Another role may have given up behind the last product: operands and tensor memory stay until all of them have completed.
    if (tid == kSoftmaxThreads + kUnpackThreads) {
        mbar_drain(bar_drain, 0);
        mbar_drain(bar_drain + 8, 0);
        Report& report = k.reports[blockIdx.x];
        report.gave_up = *abort_flag != 0;
#pragma unroll
        for (int i = 0; i < kRows / 32; ++i) report.rows[i] = anew[i] | anew[kRows / 32 + i];
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kThreads / 32 - 1) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmem);
    }
}

// Row r of head h of sample b by one warp, from the cache, in fp32: a lane has a token of a block for its logit, and element `lane` of every
// group for the output.  (All 512 rows of 32 heads, 4000 tokens: 19.7 ms, 0.11 where fp16 holds them.)
template <int D>
__device__ __noinline__ void row_anew(const AttArgs& a, int b, int h, int r, float* q) {
    using L = CacheBlock<D>;
    constexpr int G = L::G;
    constexpr float kHeadroom = 24.f;                      // (weights below 2^-24: sums with values at the end of the range hold)
    const int lane = threadIdx.x & 31, tq = quotient(r, a.R), hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
    const int len = a.cache_len ? max(0, min(__ldcg(a.cache_len + b), a.Ncap)) : a.Ncap, limit = a.causal ? max(0, len - a.Tq + tq + 1) : len;
    const __nv_bfloat16* const src = a.io.q + b * a.io.qb + hq * a.io.qh + tq * a.io.qt;
    float total[G];
    __syncwarp();
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const float x = a.sign ? -__bfloat162float(src[g * 32 + lane]) : __bfloat162float(src[g * 32 + lane]);
        q[g * 32 + lane] = total[g] = x;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) total[g] += __shfl_xor_sync(0xffffffffu, total[g], off);
    }
    __syncwarp();
    const auto bf16_at = [](const uint8_t* p) { return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p)) << 16); };
    const uint8_t* block = a.cache + ((int64_t)b * a.H + h) * (a.Ncap / kCacheBlock) * L::kBytes;
    float top = kNoLogit, sum = 0.f, v[G] = {};
    for (int token0 = 0; token0 < limit; token0 += kCacheBlock, block += L::kBytes) {
        const int seen = min(limit - token0, kCacheBlock);
        float z = MINUS_INF;
        if (lane < seen) {
            z = 0.f;
#pragma unroll 1
            for (int g = 0; g < G; ++g) {
                float dot = 0.f;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(block + L::kKCodes + lane * (D / 2) + t * 4 * G + g * 4));
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = fmaf((float)((int)(w >> (4 * e) & 15) - 8), q[g * 32 + 8 * t + e], dot);
                }
                z = fmaf(bf16_at(block + L::kKScale + (lane * G + g) * 2), dot, z);
                float group = total[0];
#pragma unroll
                for (int i = 1; i < G; ++i)
                    if (i == g) group = total[i];
                z = fmaf(bf16_at(block + L::kKCentre + (lane * G + g) * 2), group, z);
            }
        }
        float high = z;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, off));
        const float now = fmaxf(top, fmaf(high, a.scale_log2, kHeadroom)), keep = ex2_approx(top - now), p = ex2_approx(fmaf(z, a.scale_log2, -now));
        top = now;
        sum = fmaf(sum, keep, p);
#pragma unroll
        for (int g = 0; g < G; ++g) v[g] *= keep;
#pragma unroll 4
        for (int i = 0; i < seen; ++i) {
            const float w = __shfl_sync(0xffffffffu, p, i);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t c = __ldg(reinterpret_cast<const uint16_t*>(block + L::kVCodes + i * (D / 2) + (lane / 4) * 2 * G + g * 2)) >> (4 * (lane % 4)) & 15;
                v[g] = fmaf(w, fmaf((float)((int)c - 8), bf16_at(block + L::kVScale + (i * G + g) * 2), bf16_at(block + L::kVCentre + (g * 32 + i) * 2)), v[g]);
            }
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    const bool none = sum == 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
        a.io.out[b * a.io.ob + hq * a.io.oh + tq * a.io.ot + g * 32 + lane] = __float2bfloat16_rn(none ? 0.f : v[g] / sum);
    if (a.lse && lane == 0) a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = none ? MINUS_INF : (top + __log2f(sum)) * kLn2;
}

// The pieces of a row, in their order, a warp a row; rows that are to be done anew; and the status word.
constexpr int kQuarter = kRows / 4;
template <int D>
__global__ void __launch_bounds__(128)
cache_attention_rows_join_kernel(const __grid_constant__ RowsArgs k, int ctas) {
    __shared__ float queries[4][D];
    const AttArgs& a = k.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = (int)a.R.d * a.Tq;
    constexpr int E = D / 32;                              // elements of a lane: lane E .. lane E + E - 1
    grid_dependency_wait();
    if (blockIdx.x == 0 && warp == 0) {
        bool gave_up = false;
        for (int c = lane; c < ctas; c += 32) gave_up |= k.reports[c].gave_up != 0;
        gave_up = __any_sync(0xffffffffu, gave_up);
        if (lane == 0) *a.status = gave_up ? VITCOP_ERR_TIMEOUT : VITCOP_OK;
    }
    const int segs = a.H * (int)a.RT.d, items = a.B * segs * kRows;
    if (k.splits == 1) {                                   // a CTA 32 rows at a time
        for (int item = blockIdx.x; item < items / kQuarter; item += gridDim.x) {
            const int seg = item / 4, b = seg / segs, hs = seg - b * segs, h = quotient(hs, a.RT);
            const uint32_t todo = k.reports[seg].rows[item % 4];
            for (int i = warp; i < kQuarter; i += 4)
                if (todo >> i & 1) row_anew<D>(a, b, h, (hs - h * (int)a.RT.d) * kRows + (item % 4) * kQuarter + i, queries[warp]);
        }
        return;
    }
    for (int item = blockIdx.x * 4 + warp; item < items; item += gridDim.x * 4) {
        const int seg = item / kRows, rl = item - seg * kRows, b = seg / segs, hs = seg - b * segs, h = quotient(hs, a.RT);
        const int r = (hs - h * (int)a.RT.d) * kRows + rl;
        if (r >= rows) continue;
        const float* const part = a.part + (size_t)seg * k.splits * kRows * (D + 3);
        constexpr size_t kSize = (size_t)kRows * (D + 3);
        // (lane s: piece s; each piece is a mean of its own, which counts with its share of the weights)
        static_assert(kMostSplits <= 32);
        const float* const mine = part + lane * kSize + kRows * D + rl;
        const bool there = lane < k.splits;
        const bool redo = there && (k.reports[seg * k.splits + lane].rows[rl / 32] >> (rl % 32) & 1);
        const float piece = there ? mine[0] : kNoLogit;
        float top = piece, sum = there ? mine[kRows] : 0.f, weight = there ? mine[2 * kRows] : 0.f;
        if (__any_sync(0xffffffffu, redo)) {
            row_anew<D>(a, b, h, r, queries[warp]);
            continue;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float f = ex2_approx(piece - top);
        sum *= f;
        weight *= f;
        float share = weight;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, off);
            weight += __shfl_xor_sync(0xffffffffu, weight, off);
        }
        const bool none = sum == 0.f;
        share = none ? 0.f : share / weight;
        float v[E] = {};
        for (int s = 0; s < k.splits; ++s) {
            const float w = __shfl_sync(0xffffffffu, share, s);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 x = *reinterpret_cast<const float2*>(part + s * kSize + rl * D + lane * E + e);
                v[e] = fmaf(x.x, w, v[e]);
                v[e + 1] = fmaf(x.y, w, v[e + 1]);
            }
        }
        const int tq = quotient(r, a.R), hq = h * (int)a.R.d + (r - tq * (int)a.R.d);
        uint32_t* const out = reinterpret_cast<uint32_t*>(a.io.out + b * a.io.ob + hq * a.io.oh + tq * a.io.ot + lane * E);
#pragma unroll
        for (int e = 0; e < E; e += 2) out[e / 2] = bf16x2(v[e], v[e + 1]);
        if (a.lse && lane == 0) a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = none ? MINUS_INF : (top + __log2f(sum)) * kLn2;
    }
}

struct RowsPlan {
    int RT, splits;
    int64_t ctas;
};
RowsPlan plan_of(int B, int H, int Ncap, int Tq, int Hq) {
    RowsPlan p;
    const int64_t rows = (int64_t)(Hq / H) * Tq;
    p.RT = (int)((rows + kRows - 1) / kRows);
    const int64_t segs = (int64_t)B * H * p.RT, sms = sm_count(), tiles = Ncap / kTokens;
    int64_t s = segs < sms ? sms / segs : 1;
    if (s > tiles / 4) s = tiles / 4;                      // four tiles a piece at least
    p.splits = (int)(s < 1 ? 1 : s > kMostSplits ? kMostSplits : s);
    p.ctas = segs * p.splits;
    return p;
}
size_t reports_bytes(const RowsPlan& p) { return align_up((size_t)p.ctas * sizeof(Report), 256); }

template <int D>
int launch_rows(const RowsArgs& k, const RowsPlan& p, cudaStream_t stream) {
    static DoneOnDevice done;
    int rc = allow_dynamic_smem(cache_attention_rows_kernel<D>, RowsSmem<D>::kBytes, done);
    if (rc != VITCOP_OK) return rc;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = RowsSmem<D>::kBytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    {
        KernelTimeScope timed("cache_attention_rows_kernel", stream);
        rc = record_cuda(cudaLaunchKernelEx(&cfg, cache_attention_rows_kernel<D>, k));
        if (rc != VITCOP_OK) return rc;
    }
    const int64_t segs = (int64_t)k.a.B * k.a.H * p.RT, want = segs * (p.splits > 1 ? kRows / 4 : kRows / kQuarter), most = sm_count() * (p.splits > 1 ? 16 : 4);
    cfg.gridDim = dim3((unsigned)(want < most ? want : most));
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = 0;
    KernelTimeScope timed("cache_attention_rows_join_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, cache_attention_rows_join_kernel<D>, k, (int)p.ctas));
}

}  // namespace

// Where its start (10 us of a CTA) pays, and half a tile of rows is not empty.  64 rows of 32 heads, 1800 tokens: 23.3 us here, 18.0 in tiles of
// 16; of 128 heads of 64, 300 tokens: 14.0 and 10.7; 68 rows of the same: 13.9 and 18.7; 64 of 16, 4000: 23.1 and 26.8; 448 of 8, 1500: 22.3
// and 25.7; 512 of 32, 4000: 104 and some 220.
bool rows_kernel_takes(int B, int H, int Ncap, int64_t rows, int d) {
    return d != 256 && rows > 32 && (double)B * H * rows * Ncap >= (rows <= 64 ? 6e6 : 2e6);
}

size_t rows_workspace_bytes(int B, int H, int Ncap, int d, int Tq, int Hq) {
    const RowsPlan p = plan_of(B, H, Ncap, Tq, Hq);
    return kStatusBytes + reports_bytes(p) + (p.splits > 1 ? align_up((size_t)p.ctas * kRows * (d + 3) * sizeof(float), 256) : 0);
}

int launch_cache_attention_rows(const AttArgs& args, int d, void* workspace, cudaStream_t stream) {
    const RowsPlan p = plan_of(args.B, args.H, args.Ncap, args.Tq, args.Hq);
    if (p.ctas * kRows > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    RowsArgs k;
    k.a = args;
    k.a.RT = divisor(p.RT);
    k.reports = reinterpret_cast<Report*>(static_cast<char*>(workspace) + kStatusBytes);
    k.a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kStatusBytes + reports_bytes(p));
    k.splits = p.splits;
    k.wait_ns = gram_wait_limit_ns();
    k.expire_roles = pair_expire_roles();
    return d == 64 ? launch_rows<64>(k, p, stream) : launch_rows<128>(k, p, stream);
}

}  // namespace vitcop
