// cache_api.cpp -- C ABI of the 8-bit block cache: validation, planning and
// dispatch of attn_cache_plan, attn_cache_append and attn_cache_fwd. As in
// attn_api.cpp every check runs on the host before the first HIP call, and only
// ATTN_FLAG_VALIDATE reads device memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <unordered_set>
#include <vector>

#include "../../include/attn.h"
#include "api_util.h"
#include "cache_params.h"

using attn::aligned16;
using attn::CacheAppendParams;
using attn::CacheFwdKind;
using attn::CacheFwdParams;
using attn::CachePlanParams;
using attn::CachePool;
using attn::fetch;
using attn::rows_disjoint;

namespace {

constexpr int64_t kInt32Max = INT32_MAX;
// The most key splits of a row tile (the combine kernel takes one per lane).
constexpr int64_t kMaxSplits = 64;
constexpr int64_t kChunkKeys = 64;  // keys a wavefront takes at a time

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// log2 of a supported block size, else -1.
int block_shift(int32_t size)
{
    return size == 16 ? 4 : size == 32 ? 5 : size == 64 ? 6 : size == 128 ? 7 : -1;
}

bool bad_flags(uint32_t flags) { return (flags & ~(ATTN_FLAG_VALIDATE | ATTN_FLAG_LOG)) != 0; }

// Check the pool but for its pointers, and resolve its strides.
int check_cache(const attn_cache* c, CachePool* p)
{
    if (!c) return ATTN_ERR_NULL_PTR;
    if (c->struct_size != sizeof(attn_cache)) return ATTN_ERR_ABI;
    if (c->cache_dtype != ATTN_E4M3 && c->cache_dtype != ATTN_E5M2) return ATTN_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return ATTN_ERR_UNSUPPORTED;
    p->bshift = block_shift(c->block_size);
    if (p->bshift < 0) return ATTN_ERR_UNSUPPORTED;
    if (c->num_blocks <= 0 || c->num_kv_heads <= 0) return ATTN_ERR_BAD_SHAPE;
    if (c->num_kv_heads > 65535) return ATTN_ERR_UNSUPPORTED;  // a grid axis
    const int64_t page = (int64_t)c->block_size * c->head_dim, h = c->num_kv_heads;
    const int64_t in[4] = {c->stride_k_block, c->stride_k_head, c->stride_v_block, c->stride_v_head};
    int64_t out[4];
    for (int i = 0; i < 4; ++i) {
        if (in[i] < 0) return ATTN_ERR_BAD_SHAPE;
        if (in[i] % 16) return ATTN_ERR_ALIGNMENT;
        out[i] = in[i] ? in[i] : i % 2 ? page : h * page;
    }
    for (int i = 0; i < 4; i += 2) {
        const int64_t size[2] = {c->num_blocks, h}, stride[2] = {out[i], out[i + 1]};
        if (!rows_disjoint(page, 2, size, stride)) return ATTN_ERR_BAD_SHAPE;
    }
    p->sks_b = c->stride_ks_block ? c->stride_ks_block : h;
    p->svs_b = c->stride_vs_block ? c->stride_vs_block : h;
    if (c->num_blocks > 1 && (p->sks_b < h || p->svs_b < h)) return ATTN_ERR_BAD_SHAPE;
    p->sk_b = out[0], p->sk_h = out[1], p->sv_b = out[2], p->sv_h = out[3];
    p->num_blocks = c->num_blocks;
    p->hkv = c->num_kv_heads;
    return ATTN_OK;
}

int check_cache_pointers(const attn_cache* c, CachePool* p)
{
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return ATTN_ERR_NULL_PTR;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
        return ATTN_ERR_ALIGNMENT;
    p->k = static_cast<uint8_t*>(c->k);
    p->v = static_cast<uint8_t*>(c->v);
    p->k_scale = c->k_scale;
    p->v_scale = c->v_scale;
    return ATTN_OK;
}

int launched(hipError_t err, uint32_t flags, const char* what)
{
    if (err != hipSuccess && (flags & ATTN_FLAG_LOG))
        std::fprintf(stderr, "%s: launch failed: %s\n", what, hipGetErrorString(err));
    return err == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

const char* format_name(const attn_cache* c) { return c->cache_dtype == ATTN_E4M3 ? "e4m3" : "e5m2"; }

}  // namespace

extern "C" int attn_cache_plan(const attn_cache_plan_desc* desc)
{
    if (!desc) return ATTN_ERR_NULL_PTR;
    if (desc->struct_size != sizeof(attn_cache_plan_desc)) return ATTN_ERR_ABI;
    const attn_cache_plan_desc& d = *desc;
    CachePlanParams p = {};
    p.bshift = block_shift(d.block_size);
    if (p.bshift < 0) return ATTN_ERR_UNSUPPORTED;
    if (d.batch < 0 || d.table_width < 0 || d.free_len < 0 || d.total_new < 0 || d.stride_table < 0)
        return ATTN_ERR_BAD_SHAPE;
    if (d.total_new > kInt32Max) return ATTN_ERR_UNSUPPORTED;
    p.stride_table = d.stride_table ? d.stride_table : d.table_width;
    if (d.batch > 1 && p.stride_table < d.table_width) return ATTN_ERR_BAD_SHAPE;
    if (d.flags & ~ATTN_FLAG_LOG) return ATTN_ERR_BAD_VARIANT;
    if (!d.num_free || !d.num_free_out || !d.cu_seqlens_q) return ATTN_ERR_NULL_PTR;
    if (d.batch > 0 && (!d.cached_lens || !d.new_lens || !d.seqlens_k)) return ATTN_ERR_NULL_PTR;
    if (d.batch > 0 && d.table_width > 0 && !d.block_tables) return ATTN_ERR_NULL_PTR;
    if ((d.free_len > 0 && !d.free_blocks) || (d.total_new > 0 && !d.slots)) return ATTN_ERR_NULL_PTR;
    if (d.num_free_out == d.num_free) return ATTN_ERR_BAD_SHAPE;  // read by every workgroup
    for (const void* q : {(const void*)d.cached_lens, (const void*)d.new_lens, (const void*)d.block_tables,
                          (const void*)d.free_blocks, (const void*)d.num_free, (const void*)d.cu_seqlens_q,
                          (const void*)d.seqlens_k, (const void*)d.num_free_out})
        if (!aligned(q, 4)) return ATTN_ERR_ALIGNMENT;
    if (!aligned(d.slots, 8)) return ATTN_ERR_ALIGNMENT;
    p.cached = d.cached_lens;
    p.fresh = d.new_lens;
    p.table = d.block_tables;
    p.free_blocks = d.free_blocks;
    p.num_free = d.num_free;
    p.slots = d.slots;
    p.cu = d.cu_seqlens_q;
    p.seqlens = d.seqlens_k;
    p.num_free_out = d.num_free_out;
    p.total_new = d.total_new;
    p.batch = d.batch;
    p.width = d.table_width;
    p.free_len = d.free_len;
    if (d.flags & ATTN_FLAG_LOG)
        std::fprintf(stderr, "attn_cache_plan: B=%d block %d table width %d, %lld new tokens\n", d.batch,
                     d.block_size, d.table_width, (long long)d.total_new);
    return launched(attn::launch_cache_plan(p, static_cast<hipStream_t>(d.stream)), d.flags,
                    "attn_cache_plan");
}

// ATTN_FLAG_VALIDATE of attn_cache_append: one run of ascending places per block.
static int validate_slots(const attn_cache_append_desc& d, int64_t num_slots, int bshift)
{
    std::vector<int64_t> s;
    if (!fetch(d.slots, d.total_new, static_cast<hipStream_t>(d.stream), &s)) return ATTN_ERR_LAUNCH;
    std::unordered_set<int64_t> seen;
    int64_t before = -1;  // the slot before, -1 where it names none
    for (int64_t x : s) {
        if (x < 0 || x >= num_slots) {
            before = -1;
            continue;
        }
        if (before >= 0 && x >> bshift == before >> bshift) {
            if (x != before + 1) return ATTN_ERR_BAD_SHAPE;
        } else if (!seen.insert(x >> bshift).second) {
            return ATTN_ERR_BAD_SHAPE;
        }
        before = x;
    }
    return ATTN_OK;
}

extern "C" int attn_cache_append(const void* k, const void* v, const attn_cache* cache,
                                 const attn_cache_append_desc* desc)
{
    if (!desc) return ATTN_ERR_NULL_PTR;
    if (desc->struct_size != sizeof(attn_cache_append_desc)) return ATTN_ERR_ABI;
    const attn_cache_append_desc& d = *desc;
    CacheAppendParams p = {};
    int rc = check_cache(cache, &p.pool);
    if (rc != ATTN_OK) return rc;
    if (d.dtype != ATTN_BF16 && d.dtype != ATTN_FP32) return ATTN_ERR_UNSUPPORTED;
    if (d.total_new < 0) return ATTN_ERR_BAD_SHAPE;
    if (d.total_new > kInt32Max) return ATTN_ERR_UNSUPPORTED;
    if (bad_flags(d.flags)) return ATTN_ERR_BAD_VARIANT;
    const int64_t align = d.dtype == ATTN_BF16 ? 8 : 4, D = cache->head_dim;
    const int64_t in[4] = {d.stride_k_h, d.stride_v_h, d.stride_k_s, d.stride_v_s};
    int64_t out[4];
    for (int i = 0; i < 4; ++i) {
        if (in[i] < 0) return ATTN_ERR_BAD_SHAPE;
        if (in[i] % align) return ATTN_ERR_ALIGNMENT;
        out[i] = in[i] ? in[i] : i < 2 ? D : cache->num_kv_heads * D;
    }
    if (d.total_new == 0) return ATTN_OK;
    if (!k || !v || !d.slots) return ATTN_ERR_NULL_PTR;
    rc = check_cache_pointers(cache, &p.pool);
    if (rc != ATTN_OK) return rc;
    if (!aligned16(k) || !aligned16(v) || !aligned(d.slots, 8)) return ATTN_ERR_ALIGNMENT;
    p.x[0] = k;
    p.x[1] = v;
    for (int i = 0; i < 2; ++i) {
        p.sx_h[i] = out[i];
        p.sx_s[i] = out[2 + i];
    }
    p.slots = d.slots;
    p.total_new = d.total_new;
    p.num_slots = (int64_t)cache->num_blocks << p.pool.bshift;
    // Tokens a workgroup: 4 of few (a decode step's runs, one for each wavefront), up
    // to 64 of many, most of which start no run (256 tokens of as many requests 9 us
    // with 4 and 45 with 64, 18000 tokens of 8 requests 121 and 36).
    p.group = 4;
    while (p.group < 64 && d.total_new >= 128 * (int64_t)p.group) p.group *= 2;
    if ((d.total_new + p.group - 1) / p.group * cache->num_kv_heads > kInt32Max) return ATTN_ERR_UNSUPPORTED;
    if (d.flags & ATTN_FLAG_VALIDATE) {
        rc = validate_slots(d, p.num_slots, p.pool.bshift);
        if (rc != ATTN_OK) return rc;
    }
    if (d.flags & ATTN_FLAG_LOG)
        std::fprintf(stderr, "attn_cache_append: %s -> %s D=%d Hkv=%d block %d | %lld tokens, %d a workgroup\n",
                     d.dtype == ATTN_BF16 ? "bf16" : "fp32", format_name(cache), cache->head_dim,
                     cache->num_kv_heads, cache->block_size, (long long)d.total_new, p.group);
    return launched(attn::launch_cache_append(p, cache->head_dim, cache->cache_dtype == ATTN_E5M2,
                                              d.dtype == ATTN_FP32, static_cast<hipStream_t>(d.stream)),
                    d.flags, "attn_cache_append");
}

namespace {

struct FwdShape {
    CacheFwdKind kind;
    int64_t max_q;  // longest query length; 0: nothing to compute
    int64_t flat;   // flat rows of a kv head and request, at most
};

int check_fwd(const attn_cache* cache, const attn_cache_fwd_desc& d, CacheFwdParams& p, FwdShape* s)
{
    int rc = check_cache(cache, &p.pool);
    if (rc != ATTN_OK) return rc;
    if (d.dtype != ATTN_BF16 && d.dtype != ATTN_FP32) return ATTN_ERR_UNSUPPORTED;
    if (d.batch < 0 || d.num_q_heads <= 0 || d.num_q_heads % cache->num_kv_heads != 0)
        return ATTN_ERR_BAD_SHAPE;
    if (d.mask_kind != ATTN_MASK_NONE && d.mask_kind != ATTN_MASK_CAUSAL &&
        d.mask_kind != ATTN_MASK_SLIDING_WINDOW)
        return d.mask_kind >= ATTN_MASK_PREFIX_LM && d.mask_kind <= ATTN_MASK_CAUSAL_BLOCKWISE
                   ? ATTN_ERR_UNSUPPORTED
                   : ATTN_ERR_BAD_VARIANT;
    if (d.mask_kind == ATTN_MASK_SLIDING_WINDOW && (d.window_left < -1 || d.window_right < -1))
        return ATTN_ERR_BAD_VARIANT;
    if (!std::isfinite(d.scale) || !(d.scale > 0.0f)) return ATTN_ERR_BAD_VARIANT;
    if (!std::isfinite(d.softcap) || d.softcap < 0.0f) return ATTN_ERR_BAD_VARIANT;
    if (d.softcap > 0.0f && !std::isfinite(d.scale / d.softcap * (float)(2.0 * 1.4426950408889634)))
        return ATTN_ERR_BAD_VARIANT;
    if (bad_flags(d.flags)) return ATTN_ERR_BAD_VARIANT;
    const bool packed = d.cu_seqlens_q != nullptr;
    if (packed ? d.max_seqlen_q < 0 || d.total_q < 0 : d.seqlen_q < 0) return ATTN_ERR_BAD_SHAPE;
    if (d.max_seqlen_k < 0 || d.table_width < 0 || d.stride_table < 0) return ATTN_ERR_BAD_SHAPE;
    p.stride_table = d.stride_table ? d.stride_table : d.table_width;
    if (d.batch > 1 && p.stride_table < d.table_width) return ATTN_ERR_BAD_SHAPE;
    // keys are numbered with 31 bits, those of the chunks looked at ahead included
    if ((int64_t)d.table_width << p.pool.bshift > kInt32Max - 32 * kChunkKeys) return ATTN_ERR_UNSUPPORTED;
    const int64_t max_q = packed ? std::min<int64_t>(d.max_seqlen_q, d.total_q) : d.seqlen_q;
    const int64_t D = cache->head_dim, align = d.dtype == ATTN_BF16 ? 8 : 4;
    const int64_t rows = packed ? 0 : max_q;
    const int64_t in[6] = {d.stride_q_b, d.stride_q_h, d.stride_q_s, d.stride_o_b, d.stride_o_h, d.stride_o_s};
    int64_t out[6];
    for (int i = 0; i < 6; ++i) {
        if (in[i] < 0) return ATTN_ERR_BAD_SHAPE;
        if (in[i] % align) return ATTN_ERR_ALIGNMENT;
        const int64_t usual = packed ? (i % 3 == 1 ? D : i % 3 == 2 ? d.num_q_heads * D : 0)
                                     : (i % 3 == 0   ? d.num_q_heads * rows * D
                                        : i % 3 == 1 ? rows * D
                                                     : D);
        out[i] = in[i] ? in[i] : usual;
    }
    p.sq_b = packed ? 0 : out[0], p.sq_h = out[1], p.sq_s = out[2];
    p.so_b = packed ? 0 : out[3], p.so_h = out[4], p.so_s = out[5];

    p.batch = d.batch;
    p.hq = d.num_q_heads;
    p.seqlen_q = packed ? 0 : d.seqlen_q;
    p.total_q = packed ? d.total_q : 0;
    p.width = d.table_width;
    p.wl = d.mask_kind == ATTN_MASK_SLIDING_WINDOW ? d.window_left : -1;
    p.wr = d.mask_kind == ATTN_MASK_CAUSAL           ? 0
           : d.mask_kind == ATTN_MASK_SLIDING_WINDOW ? d.window_right
                                                     : -1;
    const double log2e = 1.4426950408889634;
    p.scale_u = (float)(d.scale * log2e);
    p.softcap = d.softcap;
    p.cap_pre = d.softcap > 0.0f ? d.scale / d.softcap : 0.0f;
    p.cap_pre2 = p.cap_pre * (float)(2.0 * log2e);
    p.cap_post = (float)(d.softcap * log2e);
    const int group = d.num_q_heads / cache->num_kv_heads;
    p.div_group = make_fastdiv((uint32_t)group);
    p.div_hkv = make_fastdiv((uint32_t)cache->num_kv_heads);
    s->max_q = d.batch == 0 ? 0 : max_q;
    s->flat = s->max_q * group;
    s->kind = {cache->head_dim, cache->cache_dtype == ATTN_E5M2, d.dtype == ATTN_FP32, false, 4, 1};
    // flat rows and workgroups (of 16 rows and more) are numbered with 31 bits
    const int64_t most = packed ? d.total_q : max_q;
    if (most * group > kInt32Max || (int64_t)d.batch * d.num_q_heads > kInt32Max) return ATTN_ERR_UNSUPPORTED;
    if ((s->flat + 15) / 16 * d.batch * cache->num_kv_heads > kInt32Max) return ATTN_ERR_UNSUPPORTED;
    if (d.sched_kernel < 0 || d.sched_kernel > 2 || d.sched_splits < 0 || d.sched_splits > kMaxSplits ||
        (d.sched_waves != 0 && d.sched_waves != 4 && d.sched_waves != 8) ||
        d.sched_tiles < 0 || d.sched_tiles > (s->kind.fp32 ? 1 : 2) ||
        (d.sched_kernel == 2 && ((d.sched_waves == 8 && D == 64) || (d.sched_tiles == 1 && !s->kind.fp32))))
        return ATTN_ERR_BAD_VARIANT;
    return ATTN_OK;
}

int64_t workspace_need(const CacheFwdParams& p, int64_t D)
{
    return p.splits > 1 ? p.splits * p.ws_rows * (D + 2) * (int64_t)sizeof(float) : 0;
}

// The schedules of a call: kernel, wavefronts of a workgroup, 16-row tiles of a
// wavefront; microseconds that a launch, a round of one chunk for each wavefront
// (many rows: for the workgroup), a chunk's products and softmax on one SIMD, and
// the start of a row tile that another workgroup does not cover take, head dim 128
// and bf16; workgroups that fit the chip at once (bf16 of D = 128, of D = 64, fp32
// likewise). Fitted to 460 calls of every kind (1..4096 queries, 1..128 requests of
// equal and of uneven lengths, 200..32000 keys, D = 64 and 128, bf16 and fp32) that
// were timed under each schedule and up to 64 splits: what plan_schedule takes is
// 1.6 % over the fastest on average, 7 % at the 90th percentile, 22 % at most.
struct Schedule {
    bool many;
    int waves, tiles;
    double launch, round, tile, start;
    int slots128, slots64, slots128f, slots64f;
};
constexpr Schedule kSchedules[] = {
    {false, 4, 1, 3.75, 1.68, 1.04, 0.0, 768, 1280, 512, 768}, {false, 8, 1, 4.11, 1.77, 1.04, 0.0, 256, 512, 256, 256},
    {false, 4, 2, 7.04, 2.0, 0.82, 0.0, 512, 768, 0, 0},       {false, 8, 2, 5.11, 2.49, 0.82, 0.0, 256, 256, 0, 0},
    {true, 4, 2, 5.12, 1.56, 1.01, 0.9, 512, 768, 512, 768},   {true, 8, 2, 3.51, 1.61, 0.8, 2.24, 256, 0, 256, 0},
};

// Choose kernel, tile and key splits by the time that the model above expects: of
// the longest chain of rounds, the work of all SIMDs and the memory traffic, the
// largest and a share of the others; the dispatch of the workgroups; and the
// second launch and the partial rows of a split call. The host knows the longest
// lengths only: for a batch it takes the mean of two guesses, all requests at them
// and all at 0.6 of them. The workspace stays within a quarter of the bytes of q,
// out, K and V, or 256 MiB where that is more.
void plan_schedule(const attn_cache_fwd_desc& d, FwdShape& s, CacheFwdParams& p, bool may_split)
{
    const int64_t D = s.kind.head_dim, heads = (int64_t)p.batch * p.pool.hkv;
    const int64_t group = p.div_group.d;
    const int64_t rows = d.cu_seqlens_q ? d.total_q : (int64_t)d.batch * d.seqlen_q;
    int64_t held = (int64_t)p.width << p.pool.bshift;
    if (d.max_seqlen_k > 0) held = std::min<int64_t>(held, d.max_seqlen_k);
    const int64_t bytes = 2 * D * (rows * p.hq * (s.kind.fp32 ? 4 : 2) + held * heads);
    const int64_t limit = std::max<int64_t>(bytes / 4, (int64_t)256 << 20);
    p.ws_rows = rows * p.hq;
    const int64_t part = p.ws_rows * (D + 2) * (int64_t)sizeof(float);
    const bool d64 = D == 64, f32 = s.kind.fp32, ragged = d.cu_seqlens_q && d.batch > 1;
    double best = 1e30;
    for (const Schedule& c : kSchedules) {
        const int tiles = f32 ? 1 : c.tiles;
        const int slots = f32 ? d64 ? c.slots64f : c.slots128f : d64 ? c.slots64 : c.slots128;
        if (slots == 0) continue;
        const double round = c.round * (d64 ? 0.66 : 1.0) * (!f32 ? 1.0 : c.many ? 1.35 : 1.47);
        const double tile = c.tile * (d64 ? 0.58 : 1.0) * (!f32 ? 1.0 : c.many ? 1.35 : 1.72);
        const bool forced = d.sched_kernel || d.sched_waves || d.sched_tiles;
        if (forced) {
            if ((d.sched_kernel && c.many != (d.sched_kernel == 2)) ||
                (d.sched_waves && c.waves != d.sched_waves) || (d.sched_tiles && tiles != d.sched_tiles))
                continue;
        } else if (s.flat <= 16 ? c.many || tiles > 1 : !c.many && c.tiles == 1 && s.flat > 64 && !f32) {
            continue;  // rows that one tile holds; more than four of them, with a wider one at hand
        } else if (f32 && c.many && c.waves == 8) {
            continue;  // up to a third slower than with four (23 calls, 0.5 % faster at best)
        }
        const int64_t tile_rows = 16 * tiles * (c.many ? c.waves : 1);
        const int64_t row_tiles = (s.flat + tile_rows - 1) / tile_rows;
        int64_t keys = held;
        if (p.wl >= 0 && p.wr >= 0)
            keys = std::min<int64_t>(keys, (int64_t)p.wl + p.wr + std::min(tile_rows / group + 2, s.max_q));
        const int64_t chunks = std::max<int64_t>((keys + kChunkKeys - 1) / kChunkKeys, 1);
        const double seen = p.wl < 0 && p.wr >= 0 ? std::max(1.0, (double)chunks - (double)s.max_q / 128) : (double)chunks;
        double items = (double)(heads * row_tiles);
        if (d.cu_seqlens_q)
            items = std::min(items, p.pool.hkv * ((double)(rows * group) / (double)tile_rows + 0.5 * p.batch));
        int64_t before = 0;
        for (const int64_t n : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
            const int64_t splits = d.sched_splits && may_split ? d.sched_splits : n;
            if (splits > 1 && (!may_split || (!d.sched_splits && (splits > chunks || splits * part > limit)))) break;
            const int64_t per = (chunks + splits) / splits;  // (a chunk more: a range may begin inside one)
            if (per == before) continue;
            before = per;
            const double used = splits > 1 ? (double)((chunks + per - 1) / per) : 1.0;
            const double rounds = (double)(c.many ? per : (per + c.waves - 1) / c.waves) * round;
            double us = 0.0;
            for (const double fill : {1.0, 0.6}) {
                const double avg = std::max(1.0, fill * seen), share = splits > 1 ? 1.0 : avg / (double)chunks;
                const double parts = std::max(1.0, used * fill), turns = items * parts / slots;
                // (the turns of a split call are of one length, and the last may be part full)
                const double queue = turns <= 1 ? 1.0
                                     : splits == 1
                                         ? std::max(1.0, turns * share + (ragged ? 0.39 : 0.5))
                                         : ragged ? turns + 0.57
                                                  : 0.23 * std::ceil(turns) + 0.77 * (turns + 0.5);
                const double chain = rounds * queue + c.start * (d64 ? 0.66 : 1.0) * std::max(1.0, turns);
                const double work = items * avg * (c.many ? c.waves : 1) / 1024 * tile;
                const double memory = (double)heads * avg * (double)(kChunkKeys * 2 * D) / 9.45e6;
                const double most = std::max({chain, work, memory});
                double one = c.launch + 0.0035 * items * parts * (c.waves / 4) + most +
                             0.22 * (chain + work + memory - most);
                if (splits > 1)  // the second launch, the partial rows, and the host's time for two
                    one = std::max(one + 2.48 + 2 * parts * (double)part / 4.18e6, 10.0);
                // (uneven lengths: more is left over at the end of wide workgroups)
                us += std::max(one, 6.4) * (ragged && c.many && c.waves == 8 ? 1.12 : 1.0);
                if (p.batch == 1) {
                    us *= 2;
                    break;
                }
            }
            if (us < best) {
                best = us;
                s.kind.many_rows = c.many;
                s.kind.waves = c.waves;
                s.kind.tiles = tiles;
                p.tile_rows = (int32_t)tile_rows;
                p.row_tiles = (int32_t)row_tiles;
                p.splits = (int32_t)splits;
                p.split_chunks = splits > 1 ? (int32_t)per : 1 << 30;
                // More workgroups than fit at once, whole requests each: the longest first
                // (packed prompts 254 -> 211 and 697 -> 516 us, decode of 64 requests of up
                // to 16000 keys 233 -> 198; with the keys split, or four wavefronts of few
                // rows, finding the order costs as much as it gives).
                p.by_length = splits == 1 && items > slots && p.batch > 1 && p.batch <= 64 &&
                              (c.many || c.waves == 8);
            }
            if (d.sched_splits) break;
        }
    }
}

int validate_fwd(const attn_cache_fwd_desc& d, const CacheFwdParams& p, int64_t max_q)
{
    hipStream_t stream = static_cast<hipStream_t>(d.stream);
    std::vector<int32_t> cu, lens, row;
    if (d.cu_seqlens_q) {
        if (!fetch(d.cu_seqlens_q, (int64_t)d.batch + 1, stream, &cu)) return ATTN_ERR_LAUNCH;
        if (cu[0] < 0 || cu[(size_t)d.batch] > d.total_q) return ATTN_ERR_BAD_SHAPE;
        for (int32_t b = 0; b < d.batch; ++b) {
            const int64_t n = (int64_t)cu[(size_t)b + 1] - cu[(size_t)b];
            if (n < 0 || n > max_q) return ATTN_ERR_BAD_SHAPE;
        }
    }
    if (!fetch(d.seqlens_k, d.batch, stream, &lens)) return ATTN_ERR_LAUNCH;
    for (int32_t b = 0; b < d.batch; ++b) {
        const int64_t n = lens[(size_t)b];
        if (n < 0 || n > (int64_t)p.width << p.pool.bshift) return ATTN_ERR_BAD_SHAPE;
        const int64_t used = (n + (1 << p.pool.bshift) - 1) >> p.pool.bshift;
        if (!fetch(d.block_tables + b * p.stride_table, used, stream, &row)) return ATTN_ERR_LAUNCH;
        // (entries behind a window's left end may have been given back)
        const int64_t lq = d.cu_seqlens_q ? (int64_t)cu[(size_t)b + 1] - cu[(size_t)b] : d.seqlen_q;
        const int64_t lo = p.wl < 0 ? 0 : std::max<int64_t>(n - lq - p.wl, 0);
        for (int64_t i = lo >> p.pool.bshift; i < used; ++i)
            if (row[(size_t)i] < 0 || row[(size_t)i] >= p.pool.num_blocks) return ATTN_ERR_BAD_VARIANT;
    }
    return ATTN_OK;
}

}  // namespace

extern "C" int64_t attn_cache_workspace_bytes(const attn_cache* cache, const attn_cache_fwd_desc* desc)
{
    if (!desc) return ATTN_ERR_NULL_PTR;
    if (desc->struct_size != sizeof(attn_cache_fwd_desc)) return ATTN_ERR_ABI;
    CacheFwdParams p = {};
    FwdShape s;
    const int rc = check_fwd(cache, *desc, p, &s);
    if (rc != ATTN_OK) return rc;
    if (s.max_q == 0) return 0;
    plan_schedule(*desc, s, p, true);
    return workspace_need(p, s.kind.head_dim);
}

extern "C" int attn_cache_fwd(const void* q, void* out, float* lse, const attn_cache* cache,
                              const attn_cache_fwd_desc* desc, void* workspace, int64_t workspace_bytes)
{
    if (!desc) return ATTN_ERR_NULL_PTR;
    if (desc->struct_size != sizeof(attn_cache_fwd_desc)) return ATTN_ERR_ABI;
    const attn_cache_fwd_desc& d = *desc;
    CacheFwdParams p = {};
    FwdShape s;
    int rc = check_fwd(cache, d, p, &s);
    if (rc != ATTN_OK) return rc;
    if (s.max_q == 0) return ATTN_OK;  // nothing to compute
    if (!q || !out || !d.seqlens_k || (d.table_width > 0 && !d.block_tables)) return ATTN_ERR_NULL_PTR;
    rc = check_cache_pointers(cache, &p.pool);
    if (rc != ATTN_OK) return rc;
    const bool packed = d.cu_seqlens_q != nullptr;
    {
        const int64_t size[3] = {packed ? d.total_q : d.batch, d.num_q_heads, packed ? 1 : d.seqlen_q};
        const int64_t stride[3] = {packed ? p.so_s : p.so_b, p.so_h, p.so_s};
        if (!rows_disjoint(s.kind.head_dim, 3, size, stride)) return ATTN_ERR_BAD_SHAPE;
    }
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return ATTN_ERR_ALIGNMENT;
    for (const void* a : {(const void*)lse, (const void*)d.block_tables, (const void*)d.seqlens_k,
                          (const void*)d.cu_seqlens_q, (const void*)d.alibi_slopes})
        if (!aligned(a, 4)) return ATTN_ERR_ALIGNMENT;
    p.q = q;
    p.o = out;
    p.lse = lse;
    p.slopes = d.alibi_slopes;
    p.table = d.block_tables;
    p.seqlens = d.seqlens_k;
    p.cu_q = d.cu_seqlens_q;
    plan_schedule(d, s, p, workspace != nullptr);
    const int64_t need = workspace_need(p, s.kind.head_dim);
    if (need > workspace_bytes) {
        plan_schedule(d, s, p, false);
    } else if (need > 0) {
        p.ws_o = static_cast<float*>(workspace);
        p.ws_ml = p.ws_o + p.splits * p.ws_rows * s.kind.head_dim;
    }
    if (d.flags & ATTN_FLAG_VALIDATE) {
        rc = validate_fwd(d, p, s.max_q);
        if (rc != ATTN_OK) return rc;
    }
    if (d.flags & ATTN_FLAG_LOG)
        std::fprintf(stderr,
                     "attn_cache_fwd: %s over %s D=%d B=%d Hq=%d Hkv=%d block %d %s window (%d, %d) alibi=%d "
                     "softcap=%g | %s rows, %d wavefronts, %d rows a tile, %d tiles a kv head, key splits %d\n",
                     s.kind.fp32 ? "fp32" : "bf16", format_name(cache), s.kind.head_dim, d.batch, d.num_q_heads,
                     p.pool.hkv, cache->block_size, packed ? "packed" : "fixed-length", p.wl, p.wr,
                     p.slopes != nullptr, (double)d.softcap, s.kind.many_rows ? "many" : "few", s.kind.waves,
                     p.tile_rows, p.row_tiles, p.splits);
    hipStream_t stream = static_cast<hipStream_t>(d.stream);
    const bool d128 = s.kind.head_dim == 128;
    hipError_t err = s.kind.e5m2 ? d128 ? attn::launch_cache_fwd_e5m2_d128(p, s.kind, stream)
                                        : attn::launch_cache_fwd_e5m2_d64(p, s.kind, stream)
                     : d128      ? attn::launch_cache_fwd_e4m3_d128(p, s.kind, stream)
                                 : attn::launch_cache_fwd_e4m3_d64(p, s.kind, stream);
    if (err == hipSuccess && p.splits > 1) err = attn::launch_cache_combine(p, s.kind, stream);
    return launched(err, d.flags, "attn_cache_fwd");
}
