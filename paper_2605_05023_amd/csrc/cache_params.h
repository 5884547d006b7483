// cache_params.h -- argument blocks and host entry points of the 8-bit block
// cache kernels (layouts: include/attn.h). Filled by cache_api.cpp from
// validated descriptors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastdiv.h"

namespace attn {

// The pool, strides resolved (bytes for K and V, entries for the scales).
struct CachePool {
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    int64_t sk_b, sk_h, sv_b, sv_h, sks_b, svs_b;
    int32_t num_blocks, hkv;
    int32_t bshift;  // log2(block_size)
};

struct CachePlanParams {
    const int32_t* cached;
    const int32_t* fresh;
    int32_t* table;
    const int32_t* free_blocks;
    const int32_t* num_free;
    int64_t* slots;
    int32_t* cu;
    int32_t* seqlens;
    int32_t* num_free_out;
    int64_t stride_table, total_new;
    int32_t batch, bshift, width, free_len;
};

struct CacheAppendParams {
    CachePool pool;
    const void* x[2];           // new keys, new values
    int64_t sx_h[2], sx_s[2];   // element strides
    const int64_t* slots;
    int64_t total_new;
    int64_t num_slots;          // num_blocks << bshift
    int32_t group;              // tokens whose runs one workgroup takes
};

struct CacheFwdParams {
    CachePool pool;
    const void* q;
    void* o;
    float* lse;              // may be null
    const float* slopes;     // ALiBi slope per query head, or null
    const int32_t* table;
    const int32_t* seqlens;
    const int32_t* cu_q;     // or null: seqlen_q rows of every request
    int64_t stride_table;
    int64_t total_q;
    int64_t sq_b, sq_h, sq_s, so_b, so_h, so_s;
    int32_t batch, hq, seqlen_q, width;
    int32_t wl, wr;          // window bounds, -1 = unbounded (causal: wr = 0)
    float scale_u;           // scale * log2(e)
    float softcap;           // C, 0 = off
    float cap_pre, cap_pre2, cap_post;  // scale / C, 2 log2(e) scale / C, C log2(e)
    FastDiv div_group;       // query heads of a kv head
    FastDiv div_hkv;
    // Flat row f of a kv group is query f / group of head f % group;
    // row_tiles tiles of tile_rows flat rows for each kv group.
    int32_t row_tiles, tile_rows;
    int32_t by_length;       // longest requests first (at most 64 of them)
    // Key splits: `splits` workgroups share a row tile's chunks of 64 keys, at
    // least split_chunks each. Partials, in the order of the LSE's ws_rows rows:
    // ws_o [splits][ws_rows][D], ws_ml the same with (running max, row sum).
    int32_t splits, split_chunks;
    int64_t ws_rows;
    float* ws_o;
    float* ws_ml;
};

// Variants of the attention kernel. waves: wavefronts of a workgroup, 4 or (few
// rows) 8; tiles: 16-row tiles of a wavefront.
struct CacheFwdKind {
    int head_dim;
    bool e5m2, fp32, many_rows;
    int waves, tiles;
};

hipError_t launch_cache_plan(const CachePlanParams& p, hipStream_t stream);
hipError_t launch_cache_append(const CacheAppendParams& p, int head_dim, bool e5m2, bool fp32,
                               hipStream_t stream);
// one translation unit for each format and head dim
hipError_t launch_cache_fwd_e4m3_d128(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream);
hipError_t launch_cache_fwd_e4m3_d64(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream);
hipError_t launch_cache_fwd_e5m2_d128(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream);
hipError_t launch_cache_fwd_e5m2_d64(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream);
hipError_t launch_cache_combine(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream);

}  // namespace attn
