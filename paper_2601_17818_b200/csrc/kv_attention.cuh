// What the two kernels of the attention over the cache in 4 bits share (kv_attention.cu, kv_attention_rows.cu).
#pragma once

#include <cuda_bf16.h>

#include "f32x2.cuh"
#include "kv_cache.cuh"

namespace vitcop {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#define MINUS_INF (-__builtin_huge_valf())
constexpr float kNoLogit = -3.4e38f;                       // below every logit that is a number: nothing seen yet

// n / d for 0 <= n < 2^31 by a multiplication: with l = ceil(log2 d), mul = floor(2^(31 + l) / d) + 1 is off by less than 2^l / d parts of
// 2^(31 + l), which n < 2^31 of them do not add up to a quotient.
struct Divisor {
    uint32_t d, mul, shift;
};
inline Divisor divisor(int d) {
    int l = 0;
    while ((1ll << l) < d) ++l;
    return {(uint32_t)d, d == 1 ? 0u : (uint32_t)((1ull << (31 + l)) / (uint32_t)d + 1), (uint32_t)(l > 0 ? l - 1 : 0)};
}
__device__ __forceinline__ int quotient(int n, const Divisor& by) { return by.d == 1 ? n : (int)(__umulhi((uint32_t)n, by.mul) >> by.shift); }

struct AttArgs {
    CacheQueries io;
    const uint8_t* cache;
    const int32_t* cache_len;
    float* lse;
    int* status;
    float* part;                                           // shares: two pieces a CTA, each [8 NT][D], and maximum, sum and weight [8 NT]
    int B, Hq, H, Tq, Ncap, causal;
    Divisor R, RT;                                         // query heads of a stored one, tiles of rows
    float scale_log2;                                      // above 0: the sign is the queries'
    uint32_t sign;                                         // 0x80008000 turns it
};

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {    // 128 + c, twice
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(0x000F000Fu), "r"(0x43004300u));
    return r;
}
__device__ __forceinline__ uint32_t centred(uint32_t pair) {                                              // c - 8, twice
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(0xC308C308u));
    return r;
}
#endif

// The kernel for many query rows (tcgen05): 128 rows of a head a CTA.
bool rows_kernel_takes(int B, int H, int Ncap, int64_t rows, int d);
size_t rows_workspace_bytes(int B, int H, int Ncap, int d, int Tq, int Hq);
int launch_cache_attention_rows(const AttArgs& a, int d, void* workspace, cudaStream_t stream);

int sm_count();

}  // namespace vitcop
