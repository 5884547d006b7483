// cache_plan.hip -- blocks and slots of a step's new tokens from the requests'
// lengths (attn_cache_plan in include/attn.h states the formulas).
//
// Two prefix sums over the requests, of their new tokens and of the blocks
// they need, decide everything. One launch without a wait between workgroups:
// workgroup (x, y) adds up the lengths of the requests before its 64 itself
// (8 bytes a request, read through L2), scans its own in one wavefront, and
// its threads then walk the 64 requests' new blocks and new tokens as two flat
// ranges, finding the request of each by a binary search in LDS; the y axis
// cuts the flat ranges, so that a few long prompts fill the chip too.
// Bound by latency: launch, lengths, list of free blocks. 64 requests 5.5 us a call,
// 1000 requests with up to 128 new tokens each 5.7, most of it the host's.
#include "cache_params.h"
#include "kernel_params.h"

namespace attn {
namespace {

constexpr int NT = 256, kReqs = 64;

// Inclusive prefix sum over the wavefront, without LDS: shifts within rows of 16
// lanes, then the last lane of each row (row pair) to the rows behind it.
__device__ __forceinline__ int32_t wave_scan(int32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31
    return v;
}
__device__ __forceinline__ int32_t last_lane(int32_t v) { return __builtin_amdgcn_readlane(v, 63); }

// The sums of new tokens, and so of blocks, stay below 2^31; lengths that break
// that give wrong slots, but no access out of range.
struct Request {
    int32_t cached, fresh, need;
    bool fits;
};

__device__ __forceinline__ Request request(const CachePlanParams& p, int r)
{
    Request q;
    q.cached = max(p.cached[r], 0);
    q.fresh = max(p.fresh[r], 0);
    const int64_t b1 = (1 << p.bshift) - 1;
    const int64_t last = ((int64_t)q.cached + q.fresh + b1) >> p.bshift;
    q.fits = last <= p.width;
    q.need = q.fits ? (int32_t)(last - ((q.cached + b1) >> p.bshift)) : 0;
    return q;
}

// Largest i < n with start[i] <= x (start ascending, start[0] <= x).
__device__ __forceinline__ int find(const int32_t* start, int n, int32_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(NT) void cache_plan_kernel(CachePlanParams p)
{
    __shared__ int32_t sum[2][NT / 64];
    __shared__ int32_t tok[kReqs + 1], blk[kReqs + 1];  // prefix sums, those before included
    __shared__ int32_t held[kReqs];
    __shared__ int32_t granted[kReqs];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if constexpr (kLdsPoison) {
        if (tid < kReqs) {
            tok[tid] = blk[tid] = -1;
            held[tid] = granted[tid] = -1;
        }
        __syncthreads();
    }
    const int first = (int)blockIdx.x * kReqs, n = min(kReqs, p.batch - first);
    const bool last_x = blockIdx.x == gridDim.x - 1;
    const int32_t avail = min(max(*p.num_free, 0), p.free_len);
    Request q = {0, 0, 0, true};
    if (lane < n) q = request(p, first + lane);

    int32_t t = 0, b = 0;
#pragma unroll 4
    for (int r = tid; r < first; r += NT) {
        const Request e = request(p, r);
        t += e.fresh;
        b += e.need;
    }
    t = last_lane(wave_scan(t));
    b = last_lane(wave_scan(b));
    if (lane == 0) {
        sum[0][wave] = t;
        sum[1][wave] = b;
    }
    __syncthreads();
    if (wave == 0) {
        t = b = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            t += sum[0][w];
            b += sum[1][w];
        }
        const int32_t te = t + wave_scan(q.fresh), be = b + wave_scan(q.need);
        const bool ok = q.fits && (q.need == 0 || be <= avail);
        tok[lane + 1] = te;
        blk[lane + 1] = be;
        if (lane == 0) {
            tok[0] = t;
            blk[0] = b;
        }
        held[lane] = q.cached;
        granted[lane] = ok;
        if (blockIdx.y == 0) {
            if (lane < n) {
                p.cu[first + lane] = te - q.fresh;
                p.seqlens[first + lane] = ok ? q.cached + q.fresh : q.cached;
            }
            if (last_x) {
                int32_t taken = last_lane(be);
                if (taken > avail) {
                    // more asked for than there is: the largest prefix sum of need that
                    // some granted request reaches
                    taken = 0;
                    int32_t sofar = 0;
                    for (int r0 = 0; r0 < p.batch && sofar <= avail; r0 += 64) {
                        const int32_t need = r0 + lane < p.batch ? request(p, r0 + lane).need : 0;
                        const int32_t e = sofar + wave_scan(need);
                        int32_t best = e <= avail ? e : 0;
#pragma unroll
                        for (int d = 1; d < 64; d <<= 1) best = max(best, __shfl_xor(best, d));
                        taken = max(taken, best);
                        sofar = last_lane(e);
                    }
                }
                if (lane == 0) {
                    p.cu[p.batch] = last_lane(te);
                    *p.num_free_out = avail - taken;
                }
            }
        }
    }
    __syncthreads();
    if (n > 0) {
        const int32_t b1 = (1 << p.bshift) - 1;
        const int64_t step = (int64_t)gridDim.y * NT, at = (int64_t)blockIdx.y * NT + tid;
        // new tokens
        const int64_t tend = min((int64_t)tok[n], p.total_new);
        for (int64_t i = max(tok[0], 0) + at; i < tend; i += step) {
            const int r = find(tok, n, (int32_t)i);
            int64_t slot = -1;
            if (granted[r]) {
                const int32_t pos = held[r] + ((int32_t)i - tok[r]);
                const int32_t col = pos >> p.bshift, from = (held[r] + b1) >> p.bshift;
                const int32_t up = avail - 1 - (blk[r] + col - from);
                int32_t block = -1;
                if (col < from) {
                    if (col >= 0 && col < p.width) block = p.table[(first + r) * p.stride_table + col];
                } else if (up >= 0 && up < p.free_len) {
                    block = p.free_blocks[up];
                }
                if (block >= 0) slot = ((int64_t)block << p.bshift) + (pos & b1);
            }
            p.slots[i] = slot;
        }
        // new blocks (a refused request's lie past the free list's end)
        const int64_t bend = min(blk[n], avail);
        for (int64_t i = max(blk[0], 0) + at; i < bend; i += step) {
            const int r = find(blk, n, (int32_t)i);
            const int32_t col = ((held[r] + b1) >> p.bshift) + ((int32_t)i - blk[r]);
            if (granted[r] && col >= 0 && col < p.width)
                p.table[(first + r) * p.stride_table + col] = p.free_blocks[avail - 1 - i];
        }
    }
    if (last_x) {
        const int64_t end = n > 0 ? max(tok[n], 0) : 0;
        for (int64_t i = end + (int64_t)blockIdx.y * NT + tid; i < p.total_new;
             i += (int64_t)gridDim.y * NT)
            p.slots[i] = -1;
    }
}

}  // namespace

hipError_t launch_cache_plan(const CachePlanParams& p, hipStream_t stream)
{
    const int64_t x = p.batch > 0 ? ((int64_t)p.batch + kReqs - 1) / kReqs : 1;
    // about a token for each thread
    int64_t y = p.total_new / (x * NT) + 1;
    if (y > 256) y = 256;
    hipLaunchKernelGGL(cache_plan_kernel, dim3((unsigned)x, (unsigned)y), dim3(NT), 0, stream, p);
    return hipGetLastError();
}

}  // namespace attn
