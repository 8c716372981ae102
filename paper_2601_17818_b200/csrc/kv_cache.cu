// Rows of K and V into the cache in 4 bits, and back.
//
// A group of 32 elements (one token, one head) with smallest lo and largest hi is held as s = bf16((hi - lo) / 15),
// m = bf16(lo + 8 s) and codes c = clamp(round((x - m) / s) + 8, 0, 15), which stand for m + (c - 8) s.  Both directions are
// 4 d bytes of bf16 and 1.25 d bytes of cache per row and head.  A warp takes a block of the cache, which goes through shared memory, so
// that the cache sees 16-byte pieces in a row and not the codes' two and four bytes, a scale's two.
// Writing reaches no limit: the CTAs are one wave, whose warps load, quantise (190 instructions for sixteen elements a lane, 62 % of the issue
// slots) and flush at the same time as one another.  2 x 4 heads of 128, 16512 tokens, 89 MB in 20.6 us, 4.3 TB/s.  Reading is bound by memory: 8 x 32 heads, up to 2944 tokens, 317 MB in 48.4 us, the copy rate.
#include "async_copy.cuh"
#include "f32x2.cuh"
#include "kv_cache.cuh"

namespace vitcop {
namespace {

constexpr int kCacheWarps = 4;

struct Group {
    float s, m;                                            // bf16 values
};

__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
__device__ __forceinline__ uint32_t as_u32(__nv_bfloat162 v) { return *reinterpret_cast<uint32_t*>(&v); }

// The nearest bf16 (ties to even), as fp32.
__device__ __forceinline__ float rounded(float x) { return bf16lo(as_u32(__floats2bfloat162_rn(x, x))); }

// Scale and centre of the group whose sixteen elements each of two neighbouring lanes holds.
__device__ __forceinline__ Group group_of(const uint4 (&x)[2]) {
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    __nv_bfloat162 lo2 = as_bf162(w[0]), hi2 = lo2;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo2 = __hmin2_nan(lo2, as_bf162(w[i]));
        hi2 = __hmax2_nan(hi2, as_bf162(w[i]));
    }
    // smallest, and the largest with its sign turned: one minimum of both
    uint32_t both = as_u32(__hmin2_nan(as_bf162(__byte_perm(as_u32(lo2), as_u32(hi2) ^ 0x80008000u, 0x5410)),
                                       as_bf162(__byte_perm(as_u32(lo2), as_u32(hi2) ^ 0x80008000u, 0x7632))));
    both = as_u32(__hmin2_nan(as_bf162(both), as_bf162(__shfl_xor_sync(0xffffffffu, both, 1))));
    const float lo = bf16lo(both), hi = -bf16hi(both);
    Group g;
    const float range = hi - lo;                           // NaN or infinite where an element is
    // range / 15 with a product by the reciprocal and what is left of it (Markstein's way); exact up to the rounding to bf16: a quotient
    // in the middle of two bf16 has a remainder of 0, and hi - lo needs more than 24 bits only where lo or hi is below the
    // other's last place, far from any middle
    const float fifteenth = 1.f / 15.f, q = range * fifteenth;
    g.s = rounded(fmaf(fmaf(-15.f, q, range), fifteenth, q));
    if (g.s < 7.888609052210118e-31f) g.s = 0.f;           // 2^-100: steps near the end of the exponents are none
    g.m = rounded(fmaf(8.f, g.s, lo));
    if (!(range < __builtin_huge_valf())) {
        g.s = __int_as_float(0x7fc00000);
        g.m = 0.f;
    }
    return g;
}

// Elements that are no zeros, but below 2^-16 of the centre, become 2^-16 of it.  Those are the ones whose x - m fp32 does not hold; it matters
// where m is an odd number of half steps, and the element's sign says on which side of the border between two codes x - m is.  (An element that far
// below m is in the group's range only if |m| <= 8.5 s.  m / s, a quotient of two numbers of 8 bits, then is such a border or 2^-10 and more away
// from the next, and 2^-16 |m| is less than 2^-12 s.)
__device__ __forceinline__ void raise_small(uint4 (&x)[2], float m) {
    const __nv_bfloat162 least = __float2bfloat162_rn(fabsf(m) * 0x1p-16f), zero = __float2bfloat162_rn(0.f);
    const auto raise = [&](uint32_t& w) {
        const uint32_t large = as_u32(__hmax2(as_bf162(w & 0x7FFF7FFFu), least));
        w = (large | (w & 0x80008000u)) & __hne2_mask(as_bf162(w), zero);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        raise(x[i].x);
        raise(x[i].y);
        raise(x[i].z);
        raise(x[i].w);
    }
}

// Codes of eight elements.  x - m is exact where it matters (above); its product with the reciprocal is off by a few units in the last place, and what that
// leaves of x - m, exact too, brings the quotient to the nearest there is (Markstein's way): one that is a whole number and a half comes
// out as that, and the sum with 1.5 * 2^23 rounds it to the even side.
__device__ __forceinline__ uint32_t codes_of(const uint4& x, const Group& g, float inv) {
    constexpr float kMagic = 12582912.f;                   // 1.5 * 2^23: a sum with it has the nearest whole number in its last bits
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const f32x2 m2 = pack2(-g.m, -g.m), inv2 = pack2(inv, inv), up = pack2(kMagic, kMagic), s2 = pack2(-g.s, -g.s);
    float2 n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 p = add2(pack2(bf16lo(w[i]), bf16hi(w[i])), m2), q = mul2(p, inv2);
        n[i] = unpack2(add2(fma2(fma2(q, s2, p), inv2, q), up));
    }
    // (only a centre that was rounded by half a step can push the ends out of the codes' range: its last place is 2^-8 of it)
    if (fabsf(g.m) >= 64.f * g.s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = make_float2(fminf(fmaxf(n[i].x, kMagic - 8.f), kMagic + 7.f), fminf(fmaxf(n[i].y, kMagic - 8.f), kMagic + 7.f));
    }
    // the numbers carry the bits of 1.5 * 2^23, which add up to a constant; 8 more in each nibble makes the codes
    constexpr uint32_t kBits = 0x4B400000u;
    uint32_t codes = 0x88888888u;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes -= kBits << (4 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i) codes += (__float_as_uint(n[i].x) << (8 * i)) + (__float_as_uint(n[i].y) << (8 * i + 4));
    return g.s > 0.f ? codes : 0x88888888u;                // (no step, or an element that is no number)
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

// A row's bytes in a block (K or V, `half` 0 or 1): those of sixteen elements, `part` 0 or 1 of group grp.
template <int D>
__device__ __forceinline__ void put_codes(uint8_t* block, int half, int row, int grp, int part, uint4 (&x)[2]) {
    using L = CacheBlock<D>;
    constexpr int G = L::G;
    const Group g = group_of(x);
    const float inv = __fdividef(1.f, g.s);
    // (m = border s exactly, with a border between two codes: one group of normal values in 400; 2 x 4 heads of 16512 tokens 20.6 us with and without)
    const float border = rintf(fmaf(g.m, inv, -0.5f)) + 0.5f;
    if (fmaf(-border, g.s, g.m) == 0.f) raise_small(x, g.m);
    const uint32_t c[2] = {codes_of(x[0], g, inv), codes_of(x[1], g, inv)};
    const uint16_t plane = (uint16_t)(__float_as_uint(part ? g.m : g.s) >> 16);
    if (half == 0) {
        uint8_t* const at = block + L::kKCodes + row * (D / 2) + part * 8 * G + grp * 4;
        *reinterpret_cast<uint32_t*>(at) = c[0];
        *reinterpret_cast<uint32_t*>(at + 4 * G) = c[1];
        *reinterpret_cast<uint16_t*>(block + (part ? L::kKCentre : L::kKScale) + (row * G + grp) * 2) = plane;
    } else {
        uint8_t* const at = block + L::kVCodes + row * (D / 2) + part * 8 * G + grp * 2;
        *reinterpret_cast<uint16_t*>(at) = (uint16_t)c[0];
        *reinterpret_cast<uint16_t*>(at + 2 * G) = (uint16_t)(c[0] >> 16);
        *reinterpret_cast<uint16_t*>(at + 4 * G) = (uint16_t)c[1];
        *reinterpret_cast<uint16_t*>(at + 6 * G) = (uint16_t)(c[1] >> 16);
        *reinterpret_cast<uint16_t*>(block + (part ? L::kVCentre + (grp * 32 + row) * 2 : L::kVScale + (row * G + grp) * 2)) = plane;
    }
}

// Rows first .. last - 1 of a block, K if half is 0, from shared memory to the cache; the other rows' bytes are left alone.
template <int D>
__device__ __forceinline__ void flush(const uint8_t* from, uint8_t* to, int half, int first, int last, int lane) {
    using L = CacheBlock<D>;
    constexpr int G = L::G;
    const int base = half ? L::kVCodes : L::kKCodes;
    if (first == 0 && last == 32) {
#pragma unroll
        for (int i = lane; i < 20 * D / 16; i += 32) *reinterpret_cast<uint4*>(to + base + 16 * i) = *reinterpret_cast<const uint4*>(from + base + 16 * i);
        return;
    }
    for (int i = first * (D / 32) + lane; i < last * (D / 32); i += 32)
        *reinterpret_cast<uint4*>(to + base + 16 * i) = *reinterpret_cast<const uint4*>(from + base + 16 * i);
    // planes: [32][G], and [G][32] for the centres of V
    for (int i = first * G + lane; i < last * G; i += 32) {
        const int scale = base + 16 * D + 2 * i, r = i / G, centre = base + 18 * D + 2 * (half ? (i - r * G) * 32 + r : i);
        *reinterpret_cast<uint16_t*>(to + scale) = *reinterpret_cast<const uint16_t*>(from + scale);
        *reinterpret_cast<uint16_t*>(to + centre) = *reinterpret_cast<const uint16_t*>(from + centre);
    }
}

__device__ __forceinline__ uint4 ld_row(const __nv_bfloat16* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int D>
__global__ void __launch_bounds__(kCacheWarps * 32, 8)
cache_write_kernel(CacheSource src, CacheRows rows, int H, int N, int per_head, int items, const int32_t* cache_len, uint8_t* cache,
                   int Ncap, int32_t* new_len) {
    using L = CacheBlock<D>;
    constexpr int T = D / 16, U = 32 / T, kAhead = 2;      // lanes of a row, rows of the warp at a time, of which it loads two sets ahead
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % T, mine = lane / T;
    uint8_t* const image = smem + warp * L::kBytes;
    grid_dependency_wait();
    const int item = blockIdx.x * kCacheWarps + warp;
    if (item >= items) return;
    const int bh = item / per_head, j = item - bh * per_head, b = bh / H, h = bh - b * H;
    int count = 0;
    source_row(rows, b, 0, N, count);
    const int64_t start = cache_len ? max(0, __ldcg(cache_len + b)) : 0;
    if (j == 0 && h == 0 && lane == 0) new_len[b] = (int32_t)min(start + count, (int64_t)0x7fffffff);
    const int64_t blk = start / kCacheBlock + j, end = min(start + count, (int64_t)Ncap);
    if (blk * kCacheBlock >= end) return;
    const int first = (int)max(start - blk * kCacheBlock, (int64_t)0), last = (int)min(end - blk * kCacheBlock, (int64_t)kCacheBlock);
    // lane r: where row r of the block comes from
    int from = -1, unused;
    if (lane >= first && lane < last) from = source_row(rows, b, (int)(blk * kCacheBlock + lane - start), N, unused);
    const __nv_bfloat16* const K = src.K ? src.K + b * src.kb + h * src.kh + c * 16 : nullptr;
    const __nv_bfloat16* const V = src.V ? src.V + b * src.vb + h * src.vh + c * 16 : nullptr;
    for (int r0 = first / U * U; r0 < last; r0 += kAhead * U) {
        uint4 k[kAhead][2], v[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = __shfl_sync(0xffffffffu, from, (r0 + i * U + mine) & 31);
            const bool there = r0 + i * U + mine < last && row >= 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                k[i][e] = K && there ? ld_row(K + row * src.kn + 8 * e) : make_uint4(0, 0, 0, 0);
                v[i][e] = V && there ? ld_row(V + row * src.vn + 8 * e) : make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (r0 + i * U >= last) break;                 // (uniform)
            const int row = r0 + i * U + mine;             // (below 32: its bytes are written to shared memory, whoever owns them)
            if (K) put_codes<D>(image, 0, row, c / 2, c % 2, k[i]);
            if (V) put_codes<D>(image, 1, row, c / 2, c % 2, v[i]);
        }
    }
    __syncwarp();
    uint8_t* const block = cache + ((int64_t)bh * (Ncap / kCacheBlock) + blk) * L::kBytes;
    if (K) flush<D>(image, block, 0, first, last, lane);
    if (V) flush<D>(image, block, 1, first, last, lane);
}

// Eight values from eight codes: (128 + c) - 136 = c - 8 is exact in bf16, and so is the product inside the fused sum.
__device__ __forceinline__ uint4 values_of(uint32_t codes, uint32_t s2, uint32_t m2) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                          // elements i and i + 4
        asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(x[i]) : "r"((codes >> (4 * i) & 0x000F000Fu) | 0x43004300u), "r"(0xC308C308u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(x[i]) : "r"(x[i]), "r"(s2), "r"(m2));
    }
    return make_uint4(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410), __byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632));
}
__device__ __forceinline__ uint32_t twice(const uint8_t* p) { return (uint32_t)*reinterpret_cast<const uint16_t*>(p) * 0x10001u; }

template <int D>
__global__ void __launch_bounds__(kCacheWarps * 32)
cache_read_kernel(const uint8_t* cache, int H, int Ncap, const int32_t* cache_len, const int32_t* row_begin, int row_begin_uniform,
                  uint4* K_out, uint4* V_out, int N_out, int per_head, int items) {
    using L = CacheBlock<D>;
    constexpr int G = L::G, T = D / 8, U = 32 / T;
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % T, mine = lane / T, grp = c / 4, t = c % 4;
    uint8_t* const image = smem + warp * L::kBytes;
    grid_dependency_wait();
    const int item = blockIdx.x * kCacheWarps + warp;
    if (item >= items) return;
    const int bh = item / per_head, j = item - bh * per_head, b = bh / H;
    const int64_t begin = row_begin ? max(0, __ldcg(row_begin + b)) : row_begin_uniform;
    const int64_t end = min(begin + N_out, (int64_t)(cache_len ? min(__ldcg(cache_len + b), Ncap) : Ncap)), blk = begin / kCacheBlock + j;
    if (blk * kCacheBlock >= end) return;
    const int first = (int)max(begin - blk * kCacheBlock, (int64_t)0), last = (int)min(end - blk * kCacheBlock, (int64_t)kCacheBlock);
    const uint8_t* const block = cache + ((int64_t)bh * (Ncap / kCacheBlock) + blk) * L::kBytes + (K_out ? 0 : L::kVCodes);
    const uint32_t dst = smem_u32(image) + (K_out ? 0 : L::kVCodes);
    const int pieces = (K_out && V_out ? 40 : 20) * D / 16;
    for (int i = lane; i < pieces; i += 32)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 16 * i), "l"(block + 16 * i) : "memory");
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    const int64_t out = ((int64_t)bh * N_out + (blk * kCacheBlock - begin)) * T + c;
    for (int r0 = first / U * U; r0 < last; r0 += U) {
        const int row = r0 + mine;
        if (row < first || row >= last) continue;
        if (K_out) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(image + L::kKCodes + row * (D / 2) + t * 4 * G + grp * 4);
            __stcs(K_out + out + row * T, values_of(w, twice(image + L::kKScale + (row * G + grp) * 2), twice(image + L::kKCentre + (row * G + grp) * 2)));
        }
        if (V_out) {
            const uint8_t* const at = image + L::kVCodes + row * (D / 2) + grp * 2 + 4 * t * G;
            const uint32_t w = (uint32_t)*reinterpret_cast<const uint16_t*>(at) | (uint32_t)*reinterpret_cast<const uint16_t*>(at + 2 * G) << 16;
            __stcs(V_out + out + row * T, values_of(w, twice(image + L::kVScale + (row * G + grp) * 2), twice(image + L::kVCentre + (grp * 32 + row) * 2)));
        }
    }
}

inline cudaLaunchConfig_t block_config(int items, int d, cudaLaunchAttribute* attr, cudaStream_t stream) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((items + kCacheWarps - 1) / kCacheWarps));
    cfg.blockDim = dim3(kCacheWarps * 32);
    cfg.dynamicSmemBytes = (size_t)kCacheWarps * 40 * d;   // (40 KB at most)
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_allowed(true) ? 1 : 0;
    return cfg;
}
// Blocks that `rows` rows from anywhere on may lie in.
inline int64_t blocks_for(int64_t rows) { return (rows + kCacheBlock - 2) / kCacheBlock + 1; }

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
    const int64_t per_head = blocks_for(R), items = (int64_t)B * heads * per_head;
    if (items > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    CacheSource s = src;
    if (H < 1) s.K = s.V = nullptr;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = block_config((int)items, d, attr, stream);
    KernelTimeScope timed("cache_write_kernel", stream);
    auto kern = d == 64 ? cache_write_kernel<64> : d == 128 ? cache_write_kernel<128> : cache_write_kernel<256>;
    return record_cuda(cudaLaunchKernelEx(&cfg, kern, s, rows, heads, N, (int)per_head, (int)items, cache_len, static_cast<uint8_t*>(cache),
                                          Ncap, new_len));
}

int launch_cache_read(const void* cache, int B, int H, int Ncap, int d, const int32_t* cache_len, const int32_t* row_begin,
                      int row_begin_uniform, void* K_out, void* V_out, int N_out, cudaStream_t stream) {
    if (B <= 0 || H <= 0 || N_out <= 0) return VITCOP_OK;
    const int64_t rows = N_out < Ncap ? N_out : Ncap, per_head = blocks_for(rows), items = (int64_t)B * H * per_head;
    if (items > 0x7fffffff) return VITCOP_ERR_UNSUPPORTED;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = block_config((int)items, d, attr, stream);
    KernelTimeScope timed("cache_read_kernel", stream);
    auto kern = d == 64 ? cache_read_kernel<64> : d == 128 ? cache_read_kernel<128> : cache_read_kernel<256>;
    return record_cuda(cudaLaunchKernelEx(&cfg, kern, static_cast<const uint8_t*>(cache), H, Ncap, cache_len, row_begin, row_begin_uniform,
                                          static_cast<uint4*>(K_out), static_cast<uint4*>(V_out), N_out, (int)per_head, (int)items));
}

}  // namespace vitcop
