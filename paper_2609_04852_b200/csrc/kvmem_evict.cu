// Eviction by accumulated attention weight: per session, layer and KV head the tokens of a view with the largest weight
// (and the reserved first and last ones) move together, in order, into another view.
//
// evict_select_kernel: a cluster of CTAs per head, each with a contiguous share of the head's tokens, whose weights become
// 32-bit keys in shared memory (one read of the weights).  A radix select over 11 + 11 + 10 bits finds the key of the last
// token kept: per pass a histogram in shared memory, summed over the cluster through distributed shared memory.  Counts of
// kept tokens per warp and CTA then give every kept token its place, and the places go to a list: no atomic
// decides an order, so the result is the same from run to run and ties go to the lower token.
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
constexpr int kEvKeys = 48 * 1024;                 // keys a CTA holds in shared memory; a longer share is read again per pass
constexpr size_t kEvSmem = (size_t)kEvKeys * 4;
constexpr int kEvRows = 64;                        // kept tokens per CTA of the gather

// fp32 order as unsigned order: -0 and +0 alike, a NaN above every number
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
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

// one count per lane into a histogram: the bins of the first two distinct lanes are counted for the whole warp (weights that
// are still zero share a bin), the rest one by one
__device__ __forceinline__ void count_bin(int* hist, int bin, bool live) {
    const int lane = threadIdx.x & 31;
    uint32_t todo = __ballot_sync(0xffffffffu, live);
#pragma unroll
    for (int round = 0; round < 2; ++round) {
        if (todo == 0) return;
        const int lead = __ffs(todo) - 1, b = __shfl_sync(0xffffffffu, bin, lead);
        const uint32_t same = todo & __ballot_sync(0xffffffffu, bin == b);
        if (lane == lead) atomicAdd(&hist[b], __popc(same));
        todo &= ~same;
    }
    if ((todo >> lane) & 1u) atomicAdd(&hist[bin], 1);
}

__global__ void __launch_bounds__(kEvThreads)
evict_select_kernel(EvictArgs a, int32_t* ids, int2* lengths, int cluster) {
    extern __shared__ uint32_t keys[];
    __shared__ int hist[kEvBins];
    __shared__ int warp_sum[kEvWarps], warp_tie[kEvWarps], found[2], mine[2];      // mine: tokens above the bar and at it
    pdl_wait();
    pdl_trigger();
    cg::cluster_group cl = cg::this_cluster();
    const int rank = cluster > 1 ? (int)cl.block_rank() : 0;
    const int h = blockIdx.x / cluster, s = h / a.LG, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const EvictSpan e = evict_span(a, s);
    const int lo = e.sinks, n = e.T - e.recents - e.sinks;          // tokens [lo, lo + n): their weight decides
    int want = e.K - e.sinks - e.recents;
    if (tid == 0 && rank == 0 && h % a.LG == 0) lengths[s] = make_int2(e.K, e.K / a.B);
    // the CTA's share, in whole warps of 32 tokens
    const int per = ((n + cluster - 1) / cluster + 31) & ~31;
    const int b0 = min(n, rank * per), cnt = min(n, b0 + per) - b0;
    const float* w = a.mass + (size_t)h * a.cap + lo + b0;
    const bool held = cnt <= kEvKeys;
    int32_t* list = ids + (size_t)h * a.keep * a.B;
    auto key = [&](int i) { return held ? keys[i] : weight_key(w[i]); };
    auto sync_all = [&]() { if (cluster > 1) cl.sync(); else __syncthreads(); };

    // reserved tokens need no weights
    for (int i = rank * kEvThreads + tid; i < e.sinks; i += cluster * kEvThreads) list[i] = i;
    for (int i = rank * kEvThreads + tid; i < e.recents; i += cluster * kEvThreads) list[e.K - e.recents + i] = e.T - e.recents + i;

    uint32_t bar = 0;                                               // key of the last token kept, found from the top
    int ties = 0;
    if (want == n) {                                                // everything stays (the same in the whole cluster)
        for (int i = tid; i < cnt; i += kEvThreads) list[e.sinks + b0 + i] = lo + b0 + i;
    } else if (want > 0) {
        if (held)
            for (int i = tid; i < cnt; i += kEvThreads) keys[i] = weight_key(w[i]);
        __syncthreads();
        ties = want;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
            __syncthreads();
            for (int i0 = 0; i0 < cnt; i0 += kEvThreads) {
                const int i = i0 + tid;
                const uint32_t k = i < cnt ? key(i) : 0u;
                const bool live = i < cnt && (pass == 0 || ((k ^ bar) >> (shift + bits)) == 0u);
                count_bin(hist, (int)((k >> shift) & ((1u << bits) - 1u)), live);
            }
            sync_all();
            // counts of the head for the thread's two bins, highest bin first, and the bin that holds the ties-th key from the top
            int c[2] = {0, 0};
            const int bin_hi = kEvBins - 1 - 2 * tid;
            for (int r = 0; r < cluster; ++r) {
                const int* hr = cluster > 1 ? cl.map_shared_rank(hist, r) : hist;
                c[0] += hr[bin_hi];
                c[1] += hr[bin_hi - 1];
            }
            int incl = c[0] + c[1];
            for (int d = 1; d < 32; d <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += up;
            }
            if (lane == 31) warp_sum[warp] = incl;
            __syncthreads();
            int before = incl - c[0] - c[1];
            for (int i = 0; i < warp; ++i) before += warp_sum[i];
            if (before < ties && before + c[0] >= ties) { found[0] = bin_hi; found[1] = before; }
            else if (before + c[0] < ties && before + c[0] + c[1] >= ties) { found[0] = bin_hi - 1; found[1] = before + c[0]; }
            sync_all();                                             // the histograms have been read everywhere
            bar |= (uint32_t)found[0] << shift;
            ties -= found[1];
        }
        // places: tokens above the bar, and of those at it the first `ties`
        const int share = ((cnt + kEvWarps - 1) / kEvWarps + 31) & ~31;      // tokens of a warp, consecutive
        const int i_begin = min(cnt, warp * share), i_end = min(cnt, i_begin + share);
        int above = 0, at = 0;
        for (int i = i_begin + lane; i < i_end; i += 32) {
            const uint32_t k = key(i);
            above += k > bar;
            at += k == bar;
        }
        above = __reduce_add_sync(0xffffffffu, above);
        at = __reduce_add_sync(0xffffffffu, at);
        if (lane == 0) { warp_sum[warp] = above; warp_tie[warp] = at; }
        __syncthreads();
        if (tid == 0) {
            int x = 0, y = 0;
            for (int i = 0; i < kEvWarps; ++i) { x += warp_sum[i]; y += warp_tie[i]; }
            mine[0] = x;
            mine[1] = y;
        }
        sync_all();
        int before = 0, tied = 0;                                   // tokens above the bar and at it in front of this warp
        for (int r = 0; r < rank; ++r) {
            const int* m = cl.map_shared_rank(mine, r);
            before += m[0];
            tied += m[1];
        }
        for (int i = 0; i < warp; ++i) { before += warp_sum[i]; tied += warp_tie[i]; }
        for (int i0 = i_begin; i0 < i_end; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < i_end ? key(i) : 0u;
            const bool up = i < i_end && k > bar, tie = i < i_end && k == bar;
            const uint32_t um = __ballot_sync(0xffffffffu, up), tm = __ballot_sync(0xffffffffu, tie), below = (1u << lane) - 1u;
            const int t_rank = tied + __popc(tm & below);
            if (up || (tie && t_rank < ties)) list[e.sinks + before + __popc(um & below) + min(t_rank, ties)] = lo + b0 + i;
            before += __popc(um);
            tied += __popc(tm);
        }
        sync_all();                                                 // nobody leaves while its counts may be read
    }
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

cudaError_t launch_evict(const kvmem_pool& p, const EvictArgs& a, void* workspace, cudaStream_t st) {
    static PerDeviceOnce done;
    if (done.pending(p.cfg.device)) {
        const cudaError_t e = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kEvSmem);
        if (e != cudaSuccess) return e;
        done.mark(p.cfg.device);
    }
    int2* lengths = (int2*)workspace;
    int32_t* ids = a.kept ? a.kept : (int32_t*)((char*)workspace + align_up((size_t)a.ns * sizeof(int2), 256));
    const int heads = a.ns * a.LG;
    // CTAs per head: from 4,096 tokens a CTA up, at most 8, and no more than fill the SMs once
    int cluster = 1;
    while (cluster < 8 && (long long)cluster * 4096 < a.cap && heads * cluster * 2 <= p.sm_count) cluster *= 2;
    const int share = std::min((a.cap + cluster - 1) / cluster + 31, kEvKeys);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(heads * cluster));
    cfg.blockDim = dim3(kEvThreads);
    cfg.dynamicSmemBytes = (size_t)share * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = g_pdl ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, a, ids, lengths, cluster);
    if (e != cudaSuccess) return e;
    const int chunks = (int)((std::min<long long>((long long)a.keep * a.B, a.cap) + kEvRows - 1) / kEvRows);
    return launch_pdl(evict_gather_kernel, dim3((unsigned)heads * (unsigned)chunks), dim3(256), 0, st, a, (const int32_t*)ids, (const int2*)lengths, chunks);
}

}  // namespace kvmem
