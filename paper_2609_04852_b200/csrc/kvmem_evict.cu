// Eviction by accumulated attention weight: per session, layer and KV head the tokens of a view with the largest weight
// (and the reserved first and last ones) move together, in order, into another view.
//
// evict_select_kernel: a cluster of CTAs per head, each with a contiguous share of the head's tokens, whose weights become
// 32-bit keys in shared memory (one read of the weights; a reserved token's key is above all others).  A radix select over
// 11 + 11 + 10 bits finds the key of the last token kept: per pass a histogram in shared memory, whose bins that are not
// empty every CTA adds to the sums of all CTAs of the cluster (distributed shared memory; few bins are in use, so this
// moves less than reading eight histograms and takes one cluster barrier per pass).  Counts of kept tokens per warp and
// CTA then give every kept token its place, and the places go to a list: no atomic decides an order, so the result is the
// same from run to run and ties go to the lower token.
// evict_gather_kernel: rows of 256 bytes from the places in the list to consecutive rows, a half-warp per row and 16 bytes
// per lane.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "kvmem_internal.cuh"

namespace kvmem {

namespace cg = cooperative_groups;

constexpr int kEvThreads = 1024, kEvWarps = kEvThreads / 32;
constexpr int kEvBins = 2048;
constexpr int kEvCopies = 4;                       // of a histogram: lanes of a warp that meet in a bin count in their own copy
constexpr int kEvKeys = 36 * 1024;                 // keys a CTA holds in shared memory; a longer share is read again per pass
constexpr int kEvRows = 64;                        // kept tokens per CTA of the gather
constexpr uint32_t kEvReserved = 0xffffffffu, kEvNan = 0xfffffffeu, kEvZero = 0x80000000u;

// fp32 order as unsigned order: -0 and +0 alike, a NaN above every number
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return w != w ? kEvNan : k;
}

struct EvictSpan {
    int T, K, sinks, recents;                      // tokens, tokens kept, reserved ones at either end
};
__device__ __forceinline__ EvictSpan evict_span(const EvictArgs& a, int s) {
    EvictSpan e;
    e.T = (int)min((long long)max(a.n_sel[s], 0) * a.B, (long long)a.cap);
    e.K = (int)min((long long)a.keep * a.B, (long long)e.T);
    e.sinks = min(a.n_sink, e.K);
    e.recents = min(a.n_recent, e.K - e.sinks);
    return e;
}

template <int CL>
__global__ void __launch_bounds__(kEvThreads)
evict_select_kernel(EvictArgs a, int32_t* ids, int2* lengths) {
    extern __shared__ __align__(16) uint32_t dyn[];
    int (*total)[kEvBins] = reinterpret_cast<int (*)[kEvBins]>(dyn);        // [pass]: the cluster's sums
    uint32_t* keys = dyn + 3 * kEvBins;
    __shared__ __align__(16) int hist[kEvBins * kEvCopies];
    __shared__ int warp_a[kEvWarps], warp_b[kEvWarps], found[2], mine[2];             // mine: tokens above the bar and at it
    pdl_wait();
    pdl_trigger();
    cg::cluster_group cl = cg::this_cluster();
    const int rank = CL > 1 ? (int)cl.block_rank() : 0;
    const int h = blockIdx.x / CL, s = h / a.LG, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const EvictSpan e = evict_span(a, s);
    if (tid == 0 && rank == 0 && h % a.LG == 0) lengths[s] = make_int2(e.K, e.K / a.B);
    // the CTA's share of the tokens, in whole warps of 32
    const int per = ((e.T + CL - 1) / CL + 31) & ~31;
    const int b0 = min(e.T, rank * per), cnt = min(e.T, b0 + per) - b0;
    const float* w = a.mass + (size_t)h * a.cap + b0;              // 16-byte aligned: cap and b0 are multiples of 16
    const bool held = cnt <= kEvKeys;
    int32_t* list = ids + (size_t)h * a.keep * a.B;
    const int res_lo = e.sinks - b0, res_hi = e.T - e.recents - b0;          // reserved: below and from here on
    // four keys from i on, i and cnt multiples of 4
    auto read4 = [&](int i) {
        const float4 v = *reinterpret_cast<const float4*>(w + i);
        uint4 k = make_uint4(weight_key(v.x), weight_key(v.y), weight_key(v.z), weight_key(v.w));
        if (i < res_lo || i + 4 > res_hi) {
            if (i < res_lo || i >= res_hi) k.x = kEvReserved;
            if (i + 1 < res_lo || i + 1 >= res_hi) k.y = kEvReserved;
            if (i + 2 < res_lo || i + 2 >= res_hi) k.z = kEvReserved;
            if (i + 3 < res_lo || i + 3 >= res_hi) k.w = kEvReserved;
        }
        return k;
    };
    auto key4 = [&](int i) { return held ? *reinterpret_cast<const uint4*>(keys + i) : read4(i); };
    auto key1 = [&](int i) { return held ? keys[i] : i < res_lo || i >= res_hi ? kEvReserved : weight_key(w[i]); };

    if (e.K == e.T) {                                               // everything stays (the same in the whole cluster)
        for (int i = tid; i < cnt; i += kEvThreads) list[b0 + i] = b0 + i;
        return;
    }
    for (int i = tid; i < kEvBins * kEvCopies; i += kEvThreads) hist[i] = 0;
    for (int i = tid; i < kEvBins; i += kEvThreads) total[0][i] = total[1][i] = total[2][i] = 0;
    __syncthreads();
    if (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");     // the sums are clear; waited for ahead of the first push
    int* my_hist = hist + (lane & (kEvCopies - 1));
    // keys, and the first histogram on the way.  Weights that are still zero are the one tie that comes in numbers: they are
    // counted apart and reach the histograms as one sum.
    int zeros = 0;
    for (int i = 4 * tid; i < cnt; i += 4 * kEvThreads) {           // cnt is a multiple of 16
        const uint4 k4 = read4(i);
        if (held) *reinterpret_cast<uint4*>(keys + i) = k4;
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (k[u] == kEvZero) ++zeros;
            else atomicAdd(my_hist + (k[u] >> 21) * kEvCopies, 1);
        }
    }
    zeros = __reduce_add_sync(0xffffffffu, zeros);                  // the warp's
    if (zeros && lane == 0) atomicAdd(&hist[(kEvZero >> 21) * kEvCopies], zeros);
    uint32_t bar = 0;                                               // key of the last token kept, found from the top
    int ties = e.K;                                                 // how many of the keys that share bar's known bits are kept
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        if (pass > 0) {
            for (int i = tid; i < kEvBins * kEvCopies; i += kEvThreads) hist[i] = 0;
            __syncthreads();
            for (int i = 4 * tid; i < cnt; i += 4 * kEvThreads) {
                const uint4 k4 = key4(i);
                const uint32_t k[4] = {k4.x - bar, k4.y - bar, k4.z - bar, k4.w - bar};     // below 2^(shift + bits): shares the bar's bits
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if ((k[u] >> (shift + bits)) == 0u && k[u] != kEvZero - bar) atomicAdd(my_hist + (k[u] >> shift) * kEvCopies, 1);
            }
            if (zeros && lane == 0 && ((kEvZero ^ bar) >> (shift + bits)) == 0u)
                atomicAdd(&hist[((kEvZero >> shift) & ((1u << bits) - 1u)) * kEvCopies], zeros);
        }
        __syncthreads();
        if (CL > 1 && pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (int i = tid; i < kEvBins; i += kEvThreads) {
            const int4 v4 = *reinterpret_cast<const int4*>(hist + i * kEvCopies);
            const int v = (v4.x + v4.y) + (v4.z + v4.w);
            if (CL == 1) total[pass][i] = v;
            else if (v != 0) {
#pragma unroll
                for (int r = 0; r < CL; ++r) atomicAdd(cl.map_shared_rank(&total[pass][i], r), v);
            }
        }
        if (CL > 1) cl.sync(); else __syncthreads();
        // the head's counts in the thread's two bins, highest bin first, and the bin that holds the ties-th key from the top
        const int bin_hi = kEvBins - 1 - 2 * tid;
        const int2 v2 = *reinterpret_cast<const int2*>(total[pass] + bin_hi - 1);
        const int c[2] = {v2.y, v2.x};
        int incl = c[0] + c[1];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        if (lane == 31) warp_a[warp] = incl;
        __syncthreads();
        const int before = incl - c[0] - c[1] + __reduce_add_sync(0xffffffffu, lane < warp ? warp_a[lane] : 0);
        if (before < ties && before + c[0] >= ties) { found[0] = bin_hi; found[1] = before; }
        else if (before + c[0] < ties && before + c[0] + c[1] >= ties) { found[0] = bin_hi - 1; found[1] = before + c[0]; }
        __syncthreads();
        bar |= (uint32_t)found[0] << shift;
        ties -= found[1];
    }
    // places: tokens above the bar, and of those at it the first `ties`
    const int share = ((cnt + kEvWarps - 1) / kEvWarps + 127) & ~127;        // tokens of a warp, consecutive
    const int i_begin = min(cnt, warp * share), i_end = min(cnt, i_begin + share);
    int above = 0, at = 0;
    for (int i = i_begin + 4 * lane; i < i_end; i += 128) {
        const uint4 k = key4(i);
        above += (k.x > bar) + (k.y > bar) + (k.z > bar) + (k.w > bar);
        at += (k.x == bar) + (k.y == bar) + (k.z == bar) + (k.w == bar);
    }
    above = __reduce_add_sync(0xffffffffu, above);
    at = __reduce_add_sync(0xffffffffu, at);
    if (lane == 0) { warp_a[warp] = above; warp_b[warp] = at; }
    __syncthreads();
    const int wa = warp_a[lane], wb = warp_b[lane];
    if (warp == 0) {
        const int x = __reduce_add_sync(0xffffffffu, wa), y = __reduce_add_sync(0xffffffffu, wb);
        if (lane == 0) { mine[0] = x; mine[1] = y; }
    }
    // tokens above the bar and at it in front of this warp
    int before = __reduce_add_sync(0xffffffffu, lane < warp ? wa : 0), tied = __reduce_add_sync(0xffffffffu, lane < warp ? wb : 0);
    if (CL > 1) {
        cl.sync();
        const int* m = cl.map_shared_rank(mine, lane < CL ? lane : 0);
        before += __reduce_add_sync(0xffffffffu, lane < rank ? m[0] : 0);
        tied += __reduce_add_sync(0xffffffffu, lane < rank ? m[1] : 0);
    }
    if (at == 0) {                                                  // no token of this warp is at the bar: the usual case
        int to = before + min(tied, ties);
#pragma unroll 4
        for (int i0 = i_begin; i0 < i_end; i0 += 32) {
            const bool up = i0 + lane < i_end && key1(i0 + lane) > bar;
            const uint32_t um = __ballot_sync(0xffffffffu, up);
            if (up) list[to + __popc(um & ((1u << lane) - 1u))] = b0 + i0 + lane;
            to += __popc(um);
        }
    } else {
        for (int i0 = i_begin; i0 < i_end; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < i_end ? key1(i) : 0u;
            const bool up = i < i_end && k > bar, tie = i < i_end && k == bar;
            const uint32_t um = __ballot_sync(0xffffffffu, up), tm = __ballot_sync(0xffffffffu, tie), below = (1u << lane) - 1u;
            const int t_rank = tied + __popc(tm & below);
            if (up || (tie && t_rank < ties)) list[before + __popc(um & below) + min(t_rank, ties)] = b0 + i;
            before += __popc(um);
            tied += __popc(tm);
        }
    }
    if (CL > 1) cl.sync();                                          // nobody leaves while its counts may be read
}

// The sessions' lengths come from the select kernel, since n_sel may be the array that receives the new ones.
__global__ void __launch_bounds__(256)
evict_gather_kernel(EvictArgs a, const int32_t* __restrict__ ids, const int2* __restrict__ lengths, int chunks) {
    pdl_wait();
    pdl_trigger();
    const int h = blockIdx.x / chunks, s = h / a.LG, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j0 = (blockIdx.x % chunks) * kEvRows;
    const int2 len = lengths[s];
    const int K = len.x;
    if (threadIdx.x == 0 && j0 == 0 && h % a.LG == 0) a.n_sel_out[s] = len.y;
    if (j0 >= K) return;
    const int32_t* list = ids + (size_t)h * a.keep * a.B;
    const size_t src0 = (size_t)h * a.cap, dst0 = (size_t)h * a.dst_cap;
    const uint4* kv[2] = {reinterpret_cast<const uint4*>(a.view_k), reinterpret_cast<const uint4*>(a.view_v)};
    uint4* out[2] = {reinterpret_cast<uint4*>(a.dst_k), reinterpret_cast<uint4*>(a.dst_v)};
    const int sub = lane >> 4, c = lane & 15;
    // a warp takes eight consecutive rows, two at a time: eight 16-byte loads in flight per lane
    const int jw = j0 + warp * 8;
    const int my = jw + (lane & 7) < K ? list[jw + (lane & 7)] : 0;
    uint4 v[4][2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int t = __shfl_sync(0xffffffffu, my, u * 2 + sub);
        if (jw + u * 2 + sub < K) {
            v[u][0] = __ldcs(kv[0] + (src0 + t) * 16 + c);
            v[u][1] = __ldcs(kv[1] + (src0 + t) * 16 + c);
        }
    }
    if (lane < 8 && jw + lane < K) a.dst_mass[dst0 + jw + lane] = a.mass[src0 + my];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int j = jw + u * 2 + sub;
        if (j < K) {
            __stcs(out[0] + (dst0 + j) * 16 + c, v[u][0]);
            __stcs(out[1] + (dst0 + j) * 16 + c, v[u][1]);
        }
    }
}

size_t evict_workspace_bytes(const kvmem_pool_config_t& c, int n_sessions, int keep_blocks) {
    return align_up((size_t)n_sessions * sizeof(int2), 256) +
           align_up((size_t)n_sessions * c.n_layers * c.n_kv_heads * keep_blocks * c.block_tokens * 4, 256);
}

// CTAs of the gather per head
static long long evict_chunks(long long keep_tokens, int cap) { return (std::min<long long>(keep_tokens, cap) + kEvRows - 1) / kEvRows; }

bool evict_grid_fits(const kvmem_pool_config_t& c, int n_sessions, int keep_blocks, int cap_tokens) {
    const long long heads = (long long)n_sessions * c.n_layers * c.n_kv_heads;
    const long long chunks = cap_tokens ? evict_chunks((long long)keep_blocks * c.block_tokens, cap_tokens) : 1;
    return heads <= INT32_MAX / 8 && heads * chunks <= INT32_MAX;              // eight CTAs a head at most in the selection
}

template <int CL>
static cudaError_t launch_select(const kvmem_pool& p, const EvictArgs& a, int32_t* ids, int2* lengths, cudaStream_t st) {
    static PerDeviceOnce done;
    if (done.pending(p.cfg.device)) {
        const cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kEvBins + kEvKeys) * 4);
        if (e != cudaSuccess) return e;
        done.mark(p.cfg.device);
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.ns * a.LG * CL));
    cfg.blockDim = dim3(kEvThreads);
    const int share = ((a.cap + CL - 1) / CL + 31) & ~31;
    cfg.dynamicSmemBytes = (size_t)(3 * kEvBins + std::min(share, kEvKeys)) * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = g_pdl ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<CL>, a, ids, lengths);
}

cudaError_t launch_evict(const kvmem_pool& p, const EvictArgs& a, void* workspace, cudaStream_t st) {
    int2* lengths = (int2*)workspace;
    int32_t* ids = a.kept ? a.kept : (int32_t*)((char*)workspace + align_up((size_t)a.ns * sizeof(int2), 256));
    const long long heads = (long long)a.ns * a.LG;
    const int chunks = (int)evict_chunks((long long)a.keep * a.B, a.cap);
    // CTAs per head: from 2,048 tokens a CTA up, at most 8 (a portable cluster), and no more than fill the SMs once
    int cluster = 1;
    while (cluster < 8 && (long long)cluster * 2048 < a.cap && heads * cluster * 2 <= p.sm_count) cluster *= 2;
    cudaError_t e = cluster == 1 ? launch_select<1>(p, a, ids, lengths, st) : cluster == 2 ? launch_select<2>(p, a, ids, lengths, st)
                  : cluster == 4 ? launch_select<4>(p, a, ids, lengths, st) : launch_select<8>(p, a, ids, lengths, st);
    if (e != cudaSuccess) return e;
    return launch_pdl(evict_gather_kernel, dim3((unsigned)heads * (unsigned)chunks), dim3(256), 0, st, a, (const int32_t*)ids, (const int2*)lengths, chunks);
}

}  // namespace kvmem
