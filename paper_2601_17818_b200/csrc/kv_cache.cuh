// The K/V cache in 4 bits: where its bytes are (the header states the format for callers).
//
// Blocks of 32 tokens of one head, K before V, each with its codes, scales s and centres m; G = d / 32 groups of a row.  Every byte
// belongs to one token, so one can be appended without a look at its neighbours.  The order inside a row is the one in which the
// attention's matrix instructions take it: a thread of four (K) or of eight (V) reads its share of all groups at once.
#pragma once

#include <cuda_bf16.h>

#include "internal.cuh"

namespace vitcop {

constexpr int kCacheBlock = 32;                            // tokens of a block
constexpr int kCacheGroup = 32;                            // elements of a group

template <int D>
struct CacheBlock {
    static constexpr int G = D / kCacheGroup;
    static constexpr int kKCodes = 0;                      // [32 tokens][4][G][4 bytes]: eight elements of a group together
    static constexpr int kKScale = 16 * D;                 // bf16 [32][G]
    static constexpr int kKCentre = 18 * D;                // bf16 [32][G]
    static constexpr int kVCodes = 20 * D;                 // [32 tokens][8][G][2 bytes]: four elements of a group together
    static constexpr int kVScale = 36 * D;                 // bf16 [32][G]
    static constexpr int kVCentre = 38 * D;                // bf16 [G][32]
    static constexpr int kBytes = 40 * D;
};

inline size_t cache_bytes(int B, int H, int Ncap, int d) { return (size_t)B * H * (Ncap / kCacheBlock) * 40 * d; }

// Rows of K and V with strides in elements.
struct CacheSource {
    const __nv_bfloat16 *K, *V;
    int64_t kb, kh, kn, vb, vh, vn;
};
// What a compaction keeps of them; no list: the whole sequence.
struct CacheRows {
    const int32_t* seq_len;
    int vis_start;
    const int32_t* vis_len;
    int vis_len_uniform;
    const int32_t* keep_idx;
    int keep_stride;
    const int32_t* n_keep;
};
int launch_cache_write(const CacheSource& src, const CacheRows& rows, int B, int H, int N, int d, const int32_t* cache_len,
                       void* cache, int Ncap, int32_t* new_len, cudaStream_t stream);
int launch_cache_read(const void* cache, int B, int H, int Ncap, int d, const int32_t* cache_len, const int32_t* row_begin,
                      int row_begin_uniform, void* K_out, void* V_out, int N_out, cudaStream_t stream);

struct CacheQueries {
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    int64_t qb, qh, qt, ob, oh, ot;                        // strides in elements
};
size_t cache_attention_workspace_bytes(int B, int H, int Ncap, int d, int Tq, int Hq);
int launch_cache_attention(const CacheQueries& io, const void* cache, int B, int Hq, int H, int Tq, int d, int Ncap,
                           const int32_t* cache_len, float scale, bool causal, float* lse, void* workspace, cudaStream_t stream);

}  // namespace vitcop
