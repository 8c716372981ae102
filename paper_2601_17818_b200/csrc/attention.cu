// Attention over K and V in bf16, with a window and first tokens that stay visible or with a tree of drafted tokens: the kernel for few query
// rows (a token, a few drafted ones), and which kernel a call takes.
//
// The rows of a stored head are all its query heads' (i = t R + r), 16 or 32 of them a CTA.  m16n8k16 twice: logits z = q k of 16 tokens, whose
// accumulators are, as they lie, the weights' operand of the second product.  A warp has tokens of its own, 16 at a time, which it fetches
// two blocks ahead of the one it works on, with a running maximum, sum and output of its own; a row's maximum is set high above the logits and moved only when one comes
// near it.  Up to eight CTAs of a cluster share a head's tokens; warps are joined in shared memory, CTAs in that of the cluster, so that
// there is one launch and nothing in global memory between.
// Rows of V that are no numbers must not reach queries that do not see them, and 0 times NaN does: a block that is not seen by all rows is looked
// through, and one that holds any is added token by token.
// Weights enter the second product in bf16, and the output is divided by the sum of the weights as they were rounded, which takes the
// roundings' common part out.
// Bound by HBM where the tokens are many: 7 rows of 64 heads of 128, 4160 tokens each, in 25 us (0.83 of the copy rate; 64 heads more take 20 us more,
// the copy rate, so that 5 or 6 are launch, first blocks and joins).  By latency otherwise: a row of
// 32 heads, 291 tokens, 5.6 us; 25 rows, 640 tokens, 10.7; 256 rows of 32 narrow heads, some 590 tokens, 10.7 (issue slots 35 % busy).
#include "attention.cuh"

#include <algorithm>
#include <cmath>

#include "async_copy.cuh"

namespace vitcop {
namespace {

constexpr int kWarps = 4, kBlock = 16, kStages = 3, kMostParts = 8;

template <int D, int MT>
struct FewSmem {
    static constexpr int kRows = 16 * MT;
    static constexpr int kHalf = kBlock * D * 2;                       // a block's K, or V
    static constexpr int kWarp = kStages * 2 * kHalf;                  // and, behind the blocks, the warp's output [rows][D + 8]
    static constexpr int kPitch = D + 8;
    static constexpr int kQ = kWarps * kWarp;                          // [rows][D]
    static constexpr int kEnds = kQ + kRows * D * 2;                   // [kWarps + 1][3][rows]: maximum, sum, sum of rounded weights
    static constexpr int kBytes = kEnds + ((kWarps + 1) * 3 + kMostParts) * kRows * 4;     // and [rows][parts]: what they count by
    static_assert(kRows * kPitch * 4 <= kWarp);
};

// Byte of 16-byte piece c of row r of D elements: eight rows' pieces of one column lie in all banks.
template <int D>
__device__ __forceinline__ uint32_t piece_at(int r, int c) { return (uint32_t)(r * (2 * D) + ((c ^ (r & 7)) << 4)); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory, zeros where `there` is false (and nothing is read).
__device__ __forceinline__ void fetch16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
struct FewArgs {
    SeqArgs a;
    Divisor tiles, heads;                                  // tiles of rows of a head, heads of a sample
    int ctas;                                              // of a cluster
};

template <int D, int MT, bool TREE>
__global__ void __launch_bounds__(kWarps * 32)
attention_few_kernel(const __grid_constant__ FewArgs k) {
    using S = FewSmem<D, MT>;
    constexpr int kRows = S::kRows, kPieces = D / 8, NT = D / 8;
    const SeqArgs& a = k.a;
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    float* const ends = reinterpret_cast<float*>(smem + S::kEnds);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    grid_dependency_launch_dependents();
    if (blockIdx.x == 0 && tid == 0) *a.status = VITCOP_OK;

    const int rank = blockIdx.x & (k.ctas - 1), seg = blockIdx.x / k.ctas;
    const int bh = quotient(seg, k.tiles), row0 = (seg - bh * (int)k.tiles.d) * kRows, b = quotient(bh, k.heads), h = bh - b * (int)k.heads.d;
    const int R = (int)a.R.d;
    // queries, on their way before the lengths are known (rows that the sample does not have are stored nowhere)
    constexpr int kQueryPieces = kRows * kPieces / (kWarps * 32);
    uint4 query[kQueryPieces];
#pragma unroll
    for (int n = 0; n < kQueryPieces; ++n) {
        const int i = n * kWarps * 32 + tid, r = i / kPieces, c = i % kPieces;
        query[n] = make_uint4(0, 0, 0, 0);
        if (row0 + r < R * a.Tq) {
            const int t = quotient(row0 + r, a.R), hq = h * R + (row0 + r - t * R);
            query[n] = __ldcg(reinterpret_cast<const uint4*>(a.io.q + b * a.io.q_at[0] + hq * a.io.q_at[1] + t * a.io.q_at[2] + c * 8));
        }
    }
    const Sample s = sample_of(a, b);
    const int rows = min(kRows, R * s.queries - row0);     // of this CTA
    if (rows <= 0) return;                                 // (its whole cluster)
    const Span span = span_of<TREE>(a, s, quotient(row0, a.R), quotient(row0 + rows - 1, a.R));
    const int blocks_a = (span.a + kBlock - 1) / kBlock, blocks = blocks_a + (span.b1 - span.b0 + kBlock - 1) / kBlock;
    // this CTA's blocks, and of those every fourth to a warp
    const int each = blocks / k.ctas, more = blocks - each * k.ctas, first = rank * each + min(rank, more), last = first + each + (rank < more ? 1 : 0);
    const __nv_bfloat16* const Kh = a.io.K + b * a.io.k_at[0] + h * a.io.k_at[1];
    const __nv_bfloat16* const Vh = a.io.V + b * a.io.v_at[0] + h * a.io.v_at[1];
    const auto begin_of = [&](int i) { return i < blocks_a ? i * kBlock : span.b0 + (i - blocks_a) * kBlock; };
    const auto end_of = [&](int i) { return i < blocks_a ? min(span.a, (i + 1) * kBlock) : min(span.b1, span.b0 + (i - blocks_a + 1) * kBlock); };
    const uint32_t mine = base + warp * S::kWarp;
    // (a lane has 16 bytes of every kStep-th row of a block)
    constexpr int kStep = 32 / (kPieces < 32 ? kPieces : 32), kRowsALane = kBlock / kStep;
    const int my_row = lane / kPieces, my_piece = lane % kPieces;
    const __nv_bfloat16* const Kl = Kh + my_row * a.io.k_at[2] + my_piece * 8;
    const __nv_bfloat16* const Vl = Vh + my_row * a.io.v_at[2] + my_piece * 8;
    const int64_t k_step = kStep * a.io.k_at[2], v_step = kStep * a.io.v_at[2];
    const auto fetch = [&](int i, int stage) {
        if (i < last) {
            const int j0 = begin_of(i), there = end_of(i) - j0;
            const uint32_t to = mine + stage * 2 * S::kHalf;
            const __nv_bfloat16 *pk = Kl + j0 * a.io.k_at[2], *pv = Vl + j0 * a.io.v_at[2];
#pragma unroll
            for (int n = 0; n < kRowsALane; ++n) {         // (nothing is read of rows behind the last)
                const int r = n * kStep + my_row;
                fetch16(to + piece_at<D>(r, my_piece), pk, r < there);
                fetch16(to + S::kHalf + piece_at<D>(r, my_piece), pv, r < there);
                pk += k_step;
                pv += v_step;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int st = 0; st < kStages - 1; ++st) fetch(first + warp + st * kWarps, st);

    // what the four rows of this thread see (a row behind the last sees nothing)
    const auto row_seen = [&](int r) { return Seen<TREE>(a, s, b, r < rows ? quotient(row0 + r, a.R) : s.queries); };
    Seen<TREE> seen[2 * MT] = {row_seen(lane / 4), row_seen(lane / 4 + 8)};
    if constexpr (MT == 2) {
        seen[2] = row_seen(lane / 4 + 16);
        seen[3] = row_seen(lane / 4 + 24);
    }
#pragma unroll
    for (int n = 0; n < kQueryPieces; ++n) {
        const int i = n * kWarps * 32 + tid;
        const uint4 x = query[n];
        *reinterpret_cast<uint4*>(smem + S::kQ + piece_at<D>(i / kPieces, i % kPieces)) = make_uint4(x.x ^ a.sign, x.y ^ a.sign, x.z ^ a.sign, x.w ^ a.sign);
    }
    __syncthreads();
    uint32_t q[MT][D / 16][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < D / 16; ++e) ldsm4(q[m][e], base + S::kQ + piece_at<D>(m * 16 + (lane & 15), 2 * e + (lane >> 4)));

    float o[MT][NT][4] = {}, top[2 * MT], sum[2 * MT] = {}, weight[2 * MT] = {};
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) top[i] = kNoLogit;
    int stage = 0;
#pragma unroll 1
    for (int i = first + warp; i < last; i += kWarps) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        fetch(i + (kStages - 1) * kWarps, stage == 0 ? kStages - 1 : stage - 1);       // (where the last block was, which all lanes are done with)
        const uint32_t kb = mine + stage * 2 * S::kHalf, vb = kb + S::kHalf;
        stage = stage == kStages - 1 ? 0 : stage + 1;
        float z[MT][2][4] = {};
#pragma unroll
        for (int e = 0; e < D / 16; ++e) {
            uint32_t x[4];
            ldsm4(x, kb + piece_at<D>((lane >> 4) * 8 + (lane & 7), 2 * e + ((lane >> 3) & 1)));
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                mma(z[m][0], q[m][e], x[0], x[1]);
                mma(z[m][1], q[m][e], x[2], x[3]);
            }
        }
        const int j0 = begin_of(i), j1 = end_of(i);
        const bool all = j1 - j0 == kBlock && span.full(j0, j1);
        if (!all) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = j0 + n * 8 + (lane & 3) * 2 + (e & 1);
                        if (!(j < j1 && seen[2 * m + (e >> 1)](j))) z[m][n][e] = MINUS_INF;
                    }
        }
        bool passed = false;
        float high[2 * MT];
#pragma unroll
        for (int r = 0; r < 2 * MT; ++r) {
            const float(&zm)[2][4] = z[r / 2];
            const int e = (r & 1) * 2;
            float x = fmaxf(fmaxf(zm[0][e], zm[0][e + 1]), fmaxf(zm[1][e], zm[1][e + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            high[r] = x * a.scale_log2;                    // (0 times an infinite logit: no number, and none in the output)
            passed |= high[r] > top[r] - a.room;
        }
        if (__any_sync(0xffffffffu, passed)) {
#pragma unroll
            for (int r = 0; r < 2 * MT; ++r) {
                const float now = high[r] > top[r] - a.room ? high[r] + a.headroom : top[r], keep = ex2_approx(top[r] - now);
                top[r] = now;
                sum[r] *= keep;
                weight[r] *= keep;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[r / 2][n][(r & 1) * 2] *= keep;
                    o[r / 2][n][(r & 1) * 2 + 1] *= keep;
                }
            }
        }
        uint32_t p[MT][4];
#pragma unroll
        for (int r = 0; r < 2 * MT; ++r)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float* const x = &z[r / 2][n][(r & 1) * 2];
                const float p0 = ex2_approx(fmaf(x[0], a.scale_log2, -top[r])), p1 = ex2_approx(fmaf(x[1], a.scale_log2, -top[r]));
                sum[r] += p0 + p1;
                const uint32_t w = bf16x2(p0, p1);
                weight[r] += bf16lo(w) + bf16hi(w);
                p[r / 2][2 * n + (r & 1)] = w;
            }
        bool odd = false;
        if (!all) {
            uint32_t any = 0;
#pragma unroll
            for (int n = 0; n < kBlock * kPieces / 32; ++n) {
                uint32_t x[4];
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(vb + 16 * (n * 32 + lane)) : "memory");
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= (x[e] & 0x7F807F80u) + 0x00800080u;         // (an exponent of ones carries into the sign's place)
            }
            odd = __any_sync(0xffffffffu, (any & 0x80008000u) != 0);
        }
        if (!odd) {
#pragma unroll
            for (int e = 0; e < NT / 2; ++e) {
                uint32_t x[4];
                ldsm4_t(x, vb + piece_at<D>(((lane >> 3) & 1) * 8 + (lane & 7), 2 * e + (lane >> 4)));
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    mma(o[m][2 * e], p[m], x[0], x[1]);
                    mma(o[m][2 * e + 1], p[m], x[2], x[3]);
                }
            }
        } else {
#pragma unroll 1
            for (int t = 0; t < j1 - j0; ++t) {
#pragma unroll
                for (int r = 0; r < 2 * MT; ++r) {
                    const uint32_t w0 = p[r / 2][r & 1], w1 = p[r / 2][2 + (r & 1)];
                    const uint32_t w = __shfl_sync(0xffffffffu, t < 8 ? w0 : w1, (lane & ~3) | ((t & 7) >> 1));
                    if (!seen[r](j0 + t)) continue;
                    const float f = t & 1 ? bf16hi(w) : bf16lo(w);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t v;
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(vb + piece_at<D>(t, n) + (lane & 3) * 4) : "memory");
                        o[r / 2][n][(r & 1) * 2] = fmaf(f, bf16lo(v), o[r / 2][n][(r & 1) * 2]);
                        o[r / 2][n][(r & 1) * 2 + 1] = fmaf(f, bf16hi(v), o[r / 2][n][(r & 1) * 2 + 1]);
                    }
                }
            }
        }
    }
    // ---------------------------------------------------------------------- the warps' parts
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    float* const part = reinterpret_cast<float*>(smem + warp * S::kWarp);
#pragma unroll
    for (int r = 0; r < 2 * MT; ++r) {
#pragma unroll
        for (int off = 1; off < 4; off <<= 1) {
            sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], off);
            weight[r] += __shfl_xor_sync(0xffffffffu, weight[r], off);
        }
        const int row = r * 8 + lane / 4;
        if ((lane & 3) == 0) {
            ends[(warp * 3 + 0) * kRows + row] = top[r];
            ends[(warp * 3 + 1) * kRows + row] = sum[r];
            ends[(warp * 3 + 2) * kRows + row] = weight[r];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
            *reinterpret_cast<float2*>(part + row * S::kPitch + n * 8 + (lane & 3) * 2) = make_float2(o[r / 2][n][(r & 1) * 2], o[r / 2][n][(r & 1) * 2 + 1]);
    }
    __syncthreads();
    // What each part of a row counts by, a thread a row; then the sums, a thread four elements.  At first of the warps' parts, which a CTA by itself writes out
    // and others leave in the place of the first; then of the CTAs', rows in turn to each.  Where nothing weighs anything in a whole row (it sees nothing, or
    // logits of -inf alone) its first count is kNothing: the output is 0 by selection, for parts may hold 0 times a value that is no number.
    const bool alone = k.ctas == 1;
    const auto query_of = [&](int row, int& tq, int& hq) {
        const int i = row0 + row;
        tq = quotient(i, a.R);
        hq = h * R + (i - tq * R);
    };
    const auto counted = [&](float (&tops)[kMostParts], const float (&sums)[kMostParts], const float (&weights)[kMostParts], float& t, float& su, float& we) {
        t = kNoLogit;
        su = we = 0.f;
#pragma unroll
        for (int i = 0; i < kMostParts; ++i) t = fmaxf(t, tops[i]);
#pragma unroll
        for (int i = 0; i < kMostParts; ++i) {
            tops[i] = ex2_approx(tops[i] - t);
            su = fmaf(sums[i], tops[i], su);
            we = fmaf(weights[i], tops[i], we);
        }
    };
    const auto whole = [&](int row, float t, float su) {
        int tq, hq;
        query_of(row, tq, hq);
        if (a.lse) a.lse[((int64_t)b * a.Hq + hq) * a.Tq + tq] = su == 0.f ? MINUS_INF : (t + log2f(su)) * kLn2;
    };
    const auto write = [&](int row, int e, const float4& v) {
        int tq, hq;
        query_of(row, tq, hq);
        *reinterpret_cast<uint2*>(a.io.out + b * a.io.out_at[0] + hq * a.io.out_at[1] + tq * a.io.out_at[2] + e) = make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
    };
    const auto add = [](float4& v, const float4& x, float f) {
        v.x = fmaf(x.x, f, v.x);
        v.y = fmaf(x.y, f, v.y);
        v.z = fmaf(x.z, f, v.z);
        v.w = fmaf(x.w, f, v.w);
    };
    float* const all_ends = ends + kWarps * 3 * kRows;     // [3][rows] of the CTA
    float* const counts = all_ends + 3 * kRows;            // [rows][parts]
    if (tid < rows) {
        float tops[kMostParts], sums[kMostParts], weights[kMostParts], t, su, we;
#pragma unroll
        for (int w = 0; w < kMostParts; ++w) {
            tops[w] = w < kWarps ? ends[(w * 3 + 0) * kRows + tid] : kNoLogit;
            sums[w] = w < kWarps ? ends[(w * 3 + 1) * kRows + tid] : 0.f;
            weights[w] = w < kWarps ? ends[(w * 3 + 2) * kRows + tid] : 0.f;
        }
        counted(tops, sums, weights, t, su, we);
        const float inv = alone ? 1.f / we : 1.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) counts[tid * kWarps + w] = alone && su == 0.f ? kNothing : tops[w] * inv;
        if (alone) {
            whole(tid, t, su);
        } else {
            all_ends[tid] = t;
            all_ends[kRows + tid] = su;
            all_ends[2 * kRows + tid] = we;
        }
    }
    __syncthreads();
#pragma unroll 2
    for (int i = tid; i < rows * (D / 4); i += kWarps * 32) {
        const int row = i / (D / 4), e = i % (D / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) add(v, *reinterpret_cast<const float4*>(smem + w * S::kWarp + (row * S::kPitch + e) * 4), counts[row * kWarps + w]);
        if (alone) write(row, e, counts[row * kWarps] == kNothing ? make_float4(0.f, 0.f, 0.f, 0.f) : v);
        else *reinterpret_cast<float4*>(smem + (row * S::kPitch + e) * 4) = v;     // (this thread has read what was there)
    }
    if (alone) return;
    cluster_sync_all();
    const int mine_rows = (rows - rank + k.ctas - 1) / k.ctas;
    if (tid < mine_rows) {
        const int row = rank + k.ctas * tid;
        const uint32_t at = smem_u32(all_ends + row);
        float tops[kMostParts], sums[kMostParts], weights[kMostParts], t, su, we;
#pragma unroll
        for (int c = 0; c < kMostParts; ++c) {
            const uint32_t from = cluster_map(at, c < k.ctas ? c : rank);
            tops[c] = c < k.ctas ? cluster_ld(from) : kNoLogit;
            sums[c] = c < k.ctas ? cluster_ld(from + kRows * 4) : 0.f;
            weights[c] = c < k.ctas ? cluster_ld(from + kRows * 8) : 0.f;
        }
        counted(tops, sums, weights, t, su, we);
        const float inv = 1.f / we;
#pragma unroll
        for (int c = 0; c < kMostParts; ++c)
            if (c < k.ctas) counts[tid * k.ctas + c] = su == 0.f ? kNothing : tops[c] * inv;
        whole(row, t, su);
    }
    __syncthreads();
    for (int i = tid; i < mine_rows * (D / 4); i += kWarps * 32) {
        const int j = i / (D / 4), e = i % (D / 4) * 4, row = rank + k.ctas * j;
        const uint32_t at = base + (row * S::kPitch + e) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kMostParts; ++c)
            if (c < k.ctas) add(v, cluster_ld4(cluster_map(at, c)), counts[j * k.ctas + c]);
        write(row, e, counts[j * k.ctas] == kNothing ? make_float4(0.f, 0.f, 0.f, 0.f) : v);
    }
    cluster_sync_all();                                    // (the others may still be reading what this CTA has)
}

template <int D, int MT, bool TREE>
int launch_few(FewArgs k, int64_t segs, cudaStream_t stream) {
    using S = FewSmem<D, MT>;
    static DoneOnDevice done;
    const int rc = allow_dynamic_smem(attention_few_kernel<D, MT, TREE>, S::kBytes, done);
    if (rc != VITCOP_OK) return rc;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)k.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(segs * k.ctas));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 2 : 1;
    KernelTimeScope timed("attention_few_kernel", stream);
    return record_cuda(cudaLaunchKernelEx(&cfg, attention_few_kernel<D, MT, TREE>, k));
}

template <int D, int MT>
int launch_few(const FewArgs& k, int64_t segs, cudaStream_t stream) {
    return k.a.tree ? launch_few<D, MT, true>(k, segs, stream) : launch_few<D, MT, false>(k, segs, stream);
}

// Clusters of c = 1 << log CTAs that run at a time (with either mask): not SMs / c, for a cluster stays inside a group of SMs.  (Where it cannot be told: one CTA an SM.)
template <int D, int MT>
int clusters_that_run(int log) {
    static KnownOnDevice known[4];
    static DoneOnDevice done;
    constexpr int kBytes = FewSmem<D, MT>::kBytes;
    const auto allow = [] { return allow_dynamic_smem(attention_few_kernel<D, MT, false>, kBytes, done); };
    const int n = clusters_at_once(attention_few_kernel<D, MT, false>, 1 << log, kWarps * 32, kBytes, allow, known[log]);
    return n > 0 ? n : std::max(1, sm_count() >> log);
}

// How a call is shared out, and about how many us that takes: a CTA begins and ends (with a cluster's join), and in between fetches and works on four
// blocks of 16 tokens at a time, a fifth longer for each further CTA that its SM has; clusters that do not run at once come in rounds.
// Measured (in a graph; estimate in brackets), clusters of 1 / 2 / 4 / 8, over 4160 tokens: rows of 16 heads of 64 29.3 / 17.4 / 10.9 / 8.0 us (29 / 16 / 9.9 / 7.8), of 128 56.3 /
// 31.2 / 18.0 / 11.9 (52 / 28 / 16 / 12), of 256 75.4 / 41.2 / 23.4 / 27.6 (75 / 40 / 22 / 27: 15 clusters of eight run at once); of 24 heads of 128 56.4 / 31.2 / 18.0 / 12.9
// (52 / 28 / 16 / 13); of 34 heads of 256 75.7 / 41.5 / 46.5 / 43.2 (75 / 40 / 44 / 39: 33 clusters of four).  32 rows of 16 heads of 64 41.6 / 24.6 / 15.1 / 11.4 (44 / 25 / 16 / 12),
// of 128 74.7 / 42.4 / 25.1 / 17.8 (78 / 43 / 26 / 18).  25 rows of 32 heads of 128, 640 tokens: 10.7 in fours, 11.3 in eights (11.0 and 11.3).  64 rows of 32 heads of 128,
// 355 tokens 13.1 / 10.9 / 10.8 / 18.4 (13 / 11 / 10 / 18); 7 rows of 64 heads, 4160 tokens 52.6 / 30.4 / 24.9 / 29.6 (52 / 28 / 19 / 24).
struct FewPlan {
    int tile, ctas;
    int64_t tiles, segs;
    double us;
};
FewPlan few_plan(const SeqArgs& a, int d) {
    FewPlan p;
    const int64_t rows = (int64_t)a.R.d * a.Tq;
    p.tile = rows > 16 && d != 256 ? 32 : 16;
    p.tiles = (rows + p.tile - 1) / p.tile;
    p.segs = p.tiles * a.B * a.H;
    // tokens that a tile's rows may see
    int64_t span = a.N;
    if (!a.tree) span = std::min<int64_t>(span, (int64_t)a.n_sink + a.window + p.tile / (int)a.R.d + 1);
    const bool wide = p.tile == 32;
    const double rounds = (double)span / (kWarps * kBlock), begin = d == 64 ? (wide ? 4.0 : 2.5) : wide ? 6.5 : 3.5;
    const double round = d == 64 ? (wide ? 0.62 : 0.41) : d == 128 && !wide ? 0.75 : 1.1;
    const double sms = sm_count(), joins[2][4] = {{0.0, 0.25, 0.75, 2.0}, {0.0, 1.0, 1.5, 3.0}};
    p.us = 1e30;
    p.ctas = 1;
    for (int log = 0; 1 << log <= kMostParts; ++log) {
        const int at_once = d == 256 ? clusters_that_run<256, 1>(log) : d == 128 ? (wide ? clusters_that_run<128, 2>(log) : clusters_that_run<128, 1>(log))
                                                                                   : wide ? clusters_that_run<64, 2>(log) : clusters_that_run<64, 1>(log);
        const double an_sm = std::ceil((double)(std::min<int64_t>(p.segs, at_once) << log) / sms);
        const double us = std::ceil((double)p.segs / at_once) * (begin + round * (0.8 + 0.2 * an_sm) * rounds / (1 << log)) + joins[wide][log];
        if (us < p.us) {
            p.us = us;
            p.ctas = 1 << log;
        }
    }
    return p;
}

int launch_attention_few(const SeqArgs& a, int d, const FewPlan& p, cudaStream_t stream) {
    FewArgs k;
    k.a = a;
    k.ctas = p.ctas;
    const int tile = p.tile;
    const int64_t segs = p.segs;
    if (segs * k.ctas > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    k.tiles = divisor((int)p.tiles);
    k.heads = divisor(a.H);
    switch (d) {
        case 64: return tile == 32 ? launch_few<64, 2>(k, segs, stream) : launch_few<64, 1>(k, segs, stream);
        case 128: return tile == 32 ? launch_few<128, 2>(k, segs, stream) : launch_few<128, 1>(k, segs, stream);
        default: return launch_few<256, 1>(k, segs, stream);
    }
}

}  // namespace

size_t attention_workspace_bytes(int, int, int, int, int, int) { return kStatusBytes; }

int launch_attention(const SeqRows& io, int B, int Hq, int H, int Tq, int d, int N, const int32_t* cache_len, const int32_t* query_len,
                     const int64_t* tree, int window, int n_sink, float scale, float* lse, void* workspace, cudaStream_t stream) {
    SeqArgs a;
    a.io = io;
    a.cache_len = cache_len;
    a.query_len = query_len;
    a.tree = tree;
    a.lse = lse;
    a.status = static_cast<int*>(workspace);
    a.B = B;
    a.Hq = Hq;
    a.H = H;
    a.Tq = Tq;
    a.N = N;
    a.window = window;
    a.n_sink = n_sink;
    const int64_t rows = std::max<int64_t>(1, tree ? N : std::min<int64_t>(N, (int64_t)window + n_sink));
    int room = 1;
    while (rows >> room) ++room;
    a.room = (float)room;
    a.headroom = (float)(room + kSlack);
    a.R = divisor(Hq / H);
    a.scale_log2 = std::fmax(std::fabs(scale) * kLog2e, 0x1p-149f);    // (0 times the -inf of a hidden row would be no number)
    a.sign = std::signbit(scale) ? 0x80008000u : 0u;
    const FewPlan few = few_plan(a, d);
    if (tiles_kernel_us(a, d) < few.us) {
        const int rc = launch_attention_tiles(a, d, stream);
        if (rc != VITCOP_ERR_UNSUPPORTED) return rc;
    }
    return launch_attention_few(a, d, few, stream);
}

}  // namespace vitcop
