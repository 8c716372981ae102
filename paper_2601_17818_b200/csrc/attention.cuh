// What the kernels of the attention over bf16 rows share (attention.cu, attention_tiles.cu).
#pragma once

#include <cuda_bf16.h>

#include "kv_attention.cuh"

namespace vitcop {

// Weights are 2^(logit - top), top `headroom` above the largest logit there was when it was set (in powers of two): it stays until a logit comes within `room` of it.
// 2^room is more than the rows that a query may see, so that weights add up to no more than 1 and no sum is larger than V is.  Between the two lie kSlack powers of two, which few
// logits cross (with 11 of them left: 7 % more time for prompts).  The largest weight may be 2^-headroom: a product with V is off by 2^-149 then, r rows of them by
// r 2^(headroom - 149) of the output, which counts where V is below 2^-90 or so.
constexpr int kSlack = 24;

constexpr float kNothing = -1.f;                           // in place of what a part of a row counts by, where no part weighs anything

// Queries, keys, values, output: bf16, strides of samples, heads, tokens in elements.
struct SeqRows {
    const __nv_bfloat16 *q, *K, *V;
    __nv_bfloat16* out;
    int64_t q_at[3], k_at[3], v_at[3], out_at[3];
};
struct SeqArgs {
    SeqRows io;
    const int32_t *cache_len, *query_len;                  // null: N, Tq
    const int64_t* tree;                                   // null: window and sinks
    float* lse;
    int* status;
    int B, Hq, H, Tq, N, window, n_sink;
    Divisor R;                                             // query heads of a stored one
    float room, headroom;
    float scale_log2;                                      // not below 0: the sign is the queries'
    uint32_t sign;                                         // 0x80008000 turns it
};

#ifdef __CUDACC__
// Of the shared memory of a cluster's CTA.
__device__ __forceinline__ float4 cluster_ld4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// Sample b: its rows of K and V, its queries, and the row in front of the first query's own.
struct Sample {
    int len, queries, base;
};
__device__ __forceinline__ Sample sample_of(const SeqArgs& a, int b) {
    Sample s;
    s.len = a.cache_len ? max(0, min(__ldcg(a.cache_len + b), a.N)) : a.N;
    s.queries = a.query_len ? max(0, min(__ldcg(a.query_len + b), a.Tq)) : a.Tq;
    s.base = s.len - s.queries;
    return s;
}

// What a query sees: rows below `front`, and of those behind
//   window  rows lo .. p
//   tree    rows base + i with bit i set (below base + 64)
// A query that is not there, or stands in front of the first row, sees nothing: front = 0, p = -1, no bits.
template <bool TREE>
struct Seen;
template <>
struct Seen<false> {
    int front = 0, lo = 0, p = -1;
    __device__ __forceinline__ Seen() {}
    __device__ __forceinline__ Seen(const SeqArgs& a, const Sample& s, int b, int t) {
        (void)b;
        if (t >= s.queries || s.base + t < 0) return;
        p = s.base + t;
        front = min(a.n_sink, p + 1);
        lo = max(0, p - a.window + 1);                     // (not below 0: places of rows are subtracted from it)
    }
    __device__ __forceinline__ bool operator()(int j) const { return j < front || (j >= lo && j <= p); }
};
template <>
struct Seen<true> {
    int front = 0, base = 0, len = 0;
    uint64_t bits = 0;
    __device__ __forceinline__ Seen() {}
    __device__ __forceinline__ Seen(const SeqArgs& a, const Sample& s, int b, int t) {
        base = s.base;
        len = s.len;
        if (t >= s.queries || s.base + t < 0) return;
        front = max(s.base, 0);
        bits = (uint64_t)__ldcg(reinterpret_cast<const long long*>(a.tree) + (int64_t)b * a.Tq + t);
    }
    __device__ __forceinline__ bool operator()(int j) const {
        const int i = j - base;
        return j < front || (i >= 0 && j < len && (bits >> (i & 63) & 1));     // (len - base <= 64)
    }
};

// Rows that queries t0 .. t1 of a sample may see, [0, a) and [b0, b1) with a <= b0, and which of them all of these see.
struct Span {
    int a, b0, b1, all_front, all_lo, all_hi;
    // rows s .. e - 1 are seen by all
    __device__ __forceinline__ bool full(int s, int e) const { return e <= all_front || (s >= all_lo && e <= all_hi); }
};
template <bool TREE>
__device__ __forceinline__ Span span_of(const SeqArgs& a, const Sample& s, int t0, int t1) {
    Span v = {0, 0, 0, 0, 0, 0};
    t1 = min(t1, s.queries - 1);
    if (t1 < t0 || s.base + t1 < 0) return v;
    if (TREE) {
        v.b1 = s.len;
        v.all_front = max(s.base, 0);
        if (s.base + t0 < 0) v.all_front = 0;
        return v;
    }
    const int p0 = s.base + t0, p1 = s.base + t1;
    v.b1 = p1 + 1;
    v.b0 = max(0, max(p0, 0) - a.window + 1);              // (queries in front of the first row see nothing; a window may be 2^31 - 1)
    v.a = min(a.n_sink, v.b1);
    if (v.b0 <= v.a) v.a = v.b0 = 0;
    if (p0 >= 0) {
        v.all_front = min(a.n_sink, p0 + 1);
        v.all_lo = p1 - a.window + 1;
        v.all_hi = p0 + 1;
    }
    return v;
}
#endif

int launch_attention(const SeqRows& io, int B, int Hq, int H, int Tq, int d, int N, const int32_t* cache_len, const int32_t* query_len,
                     const int64_t* tree, int window, int n_sink, float scale, float* lse, void* workspace, cudaStream_t stream);
// The kernel for many query rows (tcgen05).
double tiles_kernel_us(const SeqArgs& a, int d);           // about how long it takes; without end for what it does not do
int launch_attention_tiles(const SeqArgs& a, int d, cudaStream_t stream);
size_t attention_workspace_bytes(int B, int H, int N, int d, int Tq, int Hq);

}  // namespace vitcop
