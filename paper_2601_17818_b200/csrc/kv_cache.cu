// Rows of K and V into the cache in 4 bits, and back.
//
// A group of 32 elements (one token, one head) with smallest lo and largest hi is held as s = bf16((hi - lo) / 15),
// m = bf16(lo + 8 s) and codes c = clamp(round((x - m) / s) + 8, 0, 15), which stand for m + (c - 8) s.  Both directions are
// bound by memory (4 d bytes of bf16 and 1.25 d bytes of cache per row and head): d / 8 threads take a row, 16 bytes of K and of V each.
#include "kv_cache.cuh"

namespace vitcop {
namespace {

constexpr int kRowThreads = 256;

struct Group {
    float s, m, inv;                                       // bf16 values; inv about 1 / s, 0 where there is nothing to divide
    bool bad;                                              // an element that is no finite number
};

__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }

// Scale and centre of the group whose eight elements each of four neighbouring lanes holds.
__device__ __forceinline__ Group group_of(const uint4& x) {
    __nv_bfloat162 lo2 = __hmin2_nan(__hmin2_nan(as_bf162(x.x), as_bf162(x.y)), __hmin2_nan(as_bf162(x.z), as_bf162(x.w)));
    __nv_bfloat162 hi2 = __hmax2_nan(__hmax2_nan(as_bf162(x.x), as_bf162(x.y)), __hmax2_nan(as_bf162(x.z), as_bf162(x.w)));
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
        lo2 = __hmin2_nan(lo2, __shfl_xor_sync(0xffffffffu, lo2, off));
        hi2 = __hmax2_nan(hi2, __shfl_xor_sync(0xffffffffu, hi2, off));
    }
    const float lo = __bfloat162float(__hmin_nan(lo2.x, lo2.y)), hi = __bfloat162float(__hmax_nan(hi2.x, hi2.y));
    Group g;
    const float range = hi - lo;                           // NaN or infinite where an element is
    g.bad = !(range < __builtin_huge_valf());
    // (exact up to the rounding to bf16: hi - lo of bf16 values needs more than 24 bits only where lo or hi is below the other's
    // last place, and then the quotient is nowhere near the middle of two bf16)
    g.s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(range, 15.f)));
    if (!(g.s >= 7.888609052210118e-31f)) g.s = 0.f;       // 2^-100: steps near the end of the exponents are none
    g.m = __bfloat162float(__float2bfloat16_rn(fmaf(8.f, g.s, lo)));
    g.inv = g.s > 0.f ? __frcp_rn(g.s) : 0.f;
    if (g.bad) {
        g.s = __int_as_float(0x7fc00000);
        g.m = 0.f;
        g.inv = 0.f;
    }
    return g;
}

// round((x - m) / s) + 8 in 0 .. 15, ties to even.  The product with the reciprocal is off by a few units in the last place; what is left
// of x - m (exact: k s has 13 bits) says on which side of a border it really is.
__device__ __forceinline__ uint32_t code_of(float x, const Group& g) {
    const float p = x - g.m;
    float k = rintf(p * g.inv);
    const float left = fmaf(-k, g.s, p), half = 0.5f * g.s;
    if (fabsf(left) >= half && g.s > 0.f) {
        const bool odd = (static_cast<int>(k) & 1) != 0;
        if (fabsf(left) > half || odd) k += left > 0.f ? 1.f : -1.f;
    }
    return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(k, -8.f), 7.f)) + 8);
}

__device__ __forceinline__ uint32_t codes_of(const uint4& x, const Group& g) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c |= code_of(bf16lo(w[i]), g) << (8 * i);
        c |= code_of(bf16hi(w[i]), g) << (8 * i + 4);
    }
    return g.bad ? 0x88888888u : c;
}

// Row r of the sample's new rows: its place in the source, or -1 behind the last.
__device__ __forceinline__ int source_row(const CacheRows& rows, int b, int r, int N, int& count) {
    const int L = rows.seq_len ? max(0, min(__ldcg(rows.seq_len + b), N)) : N;
    if (!rows.keep_idx) {
        count = L;
        return r < L ? r : -1;
    }
    int nv = rows.vis_len ? __ldcg(rows.vis_len + b) : rows.vis_len_uniform;
    nv = max(0, min(nv, L - rows.vis_start));
    const int nk = max(0, min(min(__ldcg(rows.n_keep + b), rows.keep_stride), nv));
    count = L - nv + nk;
    if (r >= count) return -1;
    if (r < rows.vis_start) return r;
    if (r >= rows.vis_start + nk) return r - nk + nv;
    // (a corrupt index can never leave the span)
    return rows.vis_start + max(0, min(__ldcg(rows.keep_idx + (int64_t)b * rows.keep_stride + (r - rows.vis_start)), nv - 1));
}

template <int D>
__global__ void __launch_bounds__(kRowThreads)
cache_write_kernel(CacheSource src, CacheRows rows, int H, int N, int R, int total, const int32_t* cache_len, uint8_t* cache,
                   int Ncap, int32_t* new_len) {
    using L = CacheBlock<D>;
    constexpr int G = L::G, T = D / 8;
    grid_dependency_wait();
    const int p = blockIdx.x * (kRowThreads / T) + threadIdx.x / T;
    const int c = threadIdx.x % T, grp = c / 4, t = c % 4;
    const bool on = p < total;
    const int bh = on ? p / R : 0, r = on ? p - bh * R : 0, b = bh / H, h = bh - b * H;
    int count = 0;
    const int from = source_row(rows, b, r, N, count);
    const int64_t start = cache_len ? max(0, __ldcg(cache_len + b)) : 0;
    if (on && r == 0 && h == 0 && c == 0) new_len[b] = (int32_t)min(start + count, (int64_t)0x7fffffff);
    const int64_t to = start + r;
    const bool write = on && from >= 0 && to < Ncap;
    uint4 k = {}, v = {};
    if (write && src.K) k = __ldcg(reinterpret_cast<const uint4*>(src.K + b * src.kb + h * src.kh + from * src.kn) + c);
    if (write && src.V) v = __ldcg(reinterpret_cast<const uint4*>(src.V + b * src.vb + h * src.vh + from * src.vn) + c);
    const Group gk = group_of(k), gv = group_of(v);        // (all lanes of a warp take part)
    if (!write) return;
    uint8_t* const block = cache + ((int64_t)bh * (Ncap / kCacheBlock) + to / kCacheBlock) * L::kBytes;
    const int row = (int)(to % kCacheBlock);
    if (src.K) {
        *reinterpret_cast<uint32_t*>(block + L::kKCodes + row * (D / 2) + t * 4 * G + grp * 4) = codes_of(k, gk);
        if (t < 2)
            *reinterpret_cast<__nv_bfloat16*>(block + (t ? L::kKCentre : L::kKScale) + (row * G + grp) * 2) =
                __float2bfloat16_rn(t ? gk.m : gk.s);
    }
    if (src.V) {
        const uint32_t w = codes_of(v, gv);
        uint8_t* const at = block + L::kVCodes + row * (D / 2) + grp * 2;
        *reinterpret_cast<uint16_t*>(at + (2 * t) * 2 * G) = (uint16_t)w;
        *reinterpret_cast<uint16_t*>(at + (2 * t + 1) * 2 * G) = (uint16_t)(w >> 16);
        if (t >= 2)
            *reinterpret_cast<__nv_bfloat16*>(block + (t == 3 ? L::kVCentre + (grp * 32 + row) * 2 : L::kVScale + (row * G + grp) * 2)) =
                __float2bfloat16_rn(t == 3 ? gv.m : gv.s);
    }
}

// Eight values from eight codes.
__device__ __forceinline__ uint4 values_of(uint32_t codes, float s, float m) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = fmaf((float)(int)(codes >> (8 * i) & 15u) - 8.f, s, m);
        const float b = fmaf((float)(int)(codes >> (8 * i + 4) & 15u) - 8.f, s, m);
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        o[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ float ld_bf16(const uint8_t* p) { return __uint_as_float((uint32_t)__ldcg(reinterpret_cast<const uint16_t*>(p)) << 16); }

template <int D>
__global__ void __launch_bounds__(kRowThreads)
cache_read_kernel(const uint8_t* cache, int H, int Ncap, const int32_t* cache_len, const int32_t* row_begin, int row_begin_uniform,
                  uint4* K_out, uint4* V_out, int N_out, int total) {
    using L = CacheBlock<D>;
    constexpr int G = L::G, T = D / 8;
    grid_dependency_wait();
    const int p = blockIdx.x * (kRowThreads / T) + threadIdx.x / T;
    const int c = threadIdx.x % T, grp = c / 4, t = c % 4;
    if (p >= total) return;
    const int bh = p / N_out, i = p - bh * N_out, b = bh / H;
    const int64_t from = (int64_t)(row_begin ? max(0, __ldcg(row_begin + b)) : row_begin_uniform) + i;
    if (from >= (cache_len ? min(__ldcg(cache_len + b), Ncap) : Ncap)) return;
    const uint8_t* const block = cache + ((int64_t)bh * (Ncap / kCacheBlock) + from / kCacheBlock) * L::kBytes;
    const int row = (int)(from % kCacheBlock);
    if (K_out) {
        const uint32_t w = __ldcg(reinterpret_cast<const uint32_t*>(block + L::kKCodes + row * (D / 2) + t * 4 * G + grp * 4));
        K_out[(int64_t)p * T + c] = values_of(w, ld_bf16(block + L::kKScale + (row * G + grp) * 2), ld_bf16(block + L::kKCentre + (row * G + grp) * 2));
    }
    if (V_out) {
        const uint8_t* const at = block + L::kVCodes + row * (D / 2) + grp * 2;
        const uint32_t w = (uint32_t)__ldcg(reinterpret_cast<const uint16_t*>(at + (2 * t) * 2 * G)) |
                           (uint32_t)__ldcg(reinterpret_cast<const uint16_t*>(at + (2 * t + 1) * 2 * G)) << 16;
        V_out[(int64_t)p * T + c] = values_of(w, ld_bf16(block + L::kVScale + (row * G + grp) * 2), ld_bf16(block + L::kVCentre + (grp * 32 + row) * 2));
    }
}

inline cudaLaunchConfig_t row_config(int total, int d, cudaLaunchAttribute* attr, cudaStream_t stream) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    const int per_cta = kRowThreads / (d / 8);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((total + per_cta - 1) / per_cta));
    cfg.blockDim = dim3(kRowThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    return cfg;
}

}  // namespace

int launch_cache_write(const CacheSource& src, const CacheRows& rows, int B, int H, int N, int d, const int32_t* cache_len,
                       void* cache, int Ncap, int32_t* new_len, cudaStream_t stream) {
    if (B <= 0) return VITCOP_OK;
    // rows that a sample can have at most; one at least, whose threads report the new length
    int64_t R = N;
    if (rows.keep_idx && !rows.vis_len && rows.vis_len_uniform > rows.keep_stride && rows.seq_len == nullptr)
        R = (int64_t)N - rows.vis_len_uniform + rows.keep_stride;
    R = R < Ncap ? R : Ncap;
    if (R < 1) R = 1;
    const int heads = H < 1 ? 1 : H;
    if ((int64_t)B * heads * R > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    const int total = (int)((int64_t)B * heads * R);
    CacheSource s = src;
    if (H < 1) s.K = s.V = nullptr;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = row_config(total, d, attr, stream);
    KernelTimeScope timed("cache_write_kernel", stream);
    auto kern = d == 64 ? cache_write_kernel<64> : d == 128 ? cache_write_kernel<128> : cache_write_kernel<256>;
    return record_cuda(cudaLaunchKernelEx(&cfg, kern, s, rows, heads, N, (int)R, total, cache_len, static_cast<uint8_t*>(cache), Ncap, new_len));
}

int launch_cache_read(const void* cache, int B, int H, int Ncap, int d, const int32_t* cache_len, const int32_t* row_begin,
                      int row_begin_uniform, void* K_out, void* V_out, int N_out, cudaStream_t stream) {
    if ((int64_t)B * H * N_out > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    const int total = B * H * N_out;
    if (total <= 0) return VITCOP_OK;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = row_config(total, d, attr, stream);
    KernelTimeScope timed("cache_read_kernel", stream);
    auto kern = d == 64 ? cache_read_kernel<64> : d == 128 ? cache_read_kernel<128> : cache_read_kernel<256>;
    return record_cuda(cudaLaunchKernelEx(&cfg, kern, static_cast<const uint8_t*>(cache), H, Ncap, cache_len, row_begin, row_begin_uniform,
                                          static_cast<uint4*>(K_out), static_cast<uint4*>(V_out), N_out, total));
}

}  // namespace vitcop
