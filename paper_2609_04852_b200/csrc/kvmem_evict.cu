// Eviction by accumulated attention weight: per session, layer and KV head the tokens of a view with the largest weight
// (and the reserved first and last ones) move together, in order, into another view.
// One CTA per head.  A weight's order is that of a 32-bit key; the key of the last token kept is found bit by bit, each
// a count over the head's tokens.  A second sweep gives every kept token its place (ranks by ballot and prefix sums)
// and a third copies the rows.
#include <math.h>

#include "kvmem_internal.cuh"

namespace kvmem {

constexpr int kEvThreads = 1024;

// fp32 order as unsigned order: -0 and +0 alike, a NaN above every number
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int block_sum(int v, int* red) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    int t = 0;
    for (int i = 0; i < kEvThreads / 32; ++i) t += red[i];
    return t;
}

__global__ void __launch_bounds__(kEvThreads) evict_kernel(EvictArgs a, int32_t* ids) {
    __shared__ int red[32];
    const int h = blockIdx.x, s = h / a.LG, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int T = (int)min((long long)max(a.n_sel[s], 0) * a.B, (long long)a.cap);
    const int C = a.keep * a.B, K = min(C, T);
    const int sinks = min(a.n_sink, K), recents = min(a.n_recent, K - sinks);
    const int lo = sinks, hi = T - recents;              // the tokens whose weight decides
    const int want = K - sinks - recents;
    const float* w = a.mass + (size_t)h * a.cap;
    uint32_t bar = 0;                                    // largest key that at least `want` tokens reach
    for (int bit = 31; bit >= 0 && want > 0; --bit) {
        const uint32_t c = bar | (1u << bit);
        int n = 0;
        for (int t = lo + tid; t < hi; t += kEvThreads) n += weight_key(w[t]) >= c;
        if (block_sum(n, red) >= want) bar = c;
    }
    int above = 0;
    for (int t = lo + tid; t < hi; t += kEvThreads) above += weight_key(w[t]) > bar;
    int ties = want - block_sum(above, red);             // tokens at the bar that are kept, lowest first
    int base = 0;                                        // kept so far
    for (int t0 = 0; t0 < T; t0 += kEvThreads) {
        const int t = t0 + tid;
        const bool inside = t >= lo && t < hi;
        const uint32_t k = inside ? weight_key(w[t]) : 0u;
        const bool tie = inside && want > 0 && k == bar;
        auto before = [&](bool f, int* total) {          // how many threads below this one have f
            const uint32_t b = __ballot_sync(0xffffffffu, f);
            __syncthreads();
            if (lane == 0) red[warp] = __popc(b);
            __syncthreads();
            int n = 0, all = 0;
            for (int i = 0; i < kEvThreads / 32; ++i) { if (i < warp) n += red[i]; all += red[i]; }
            *total = all;
            return n + __popc(b & ((1u << lane) - 1u));
        };
        int n_tie, n_kept;
        const int tie_rank = before(tie, &n_tie);
        const bool keep = t < T && (!inside || (want > 0 && (k > bar || (tie && tie_rank < ties))));
        const int at = base + before(keep, &n_kept);
        if (keep) ids[(size_t)h * C + at] = t;
        ties -= min(ties, n_tie);
        base += n_kept;
    }
    __syncthreads();
    for (int j = warp; j < K; j += kEvThreads / 32) {
        const int t = ids[(size_t)h * C + j];
        const size_t src = ((size_t)h * a.cap + t) * 128, dst = ((size_t)h * a.dst_cap + j) * 128;
        for (int d = lane; d < 128; d += 32) { a.dst_k[dst + d] = a.view_k[src + d]; a.dst_v[dst + d] = a.view_v[src + d]; }
        if (lane == 0) a.dst_mass[(size_t)h * a.dst_cap + j] = w[t];
    }
}

__global__ void evict_length_kernel(EvictArgs a) {
    const int s = blockIdx.x * blockDim.x + threadIdx.x;
    if (s < a.ns) a.n_sel_out[s] = min(a.keep, min(max(a.n_sel[s], 0), a.cap / a.B));
}

size_t evict_workspace_bytes(const kvmem_pool_config_t& c, int n_sessions, int keep_blocks) {
    return align_up((size_t)n_sessions * c.n_layers * c.n_kv_heads * keep_blocks * c.block_tokens * 4, 256);
}

cudaError_t launch_evict(const kvmem_pool& p, const EvictArgs& a, void* workspace, cudaStream_t st) {
    (void)p;
    evict_kernel<<<a.ns * a.LG, kEvThreads, 0, st>>>(a, a.kept ? a.kept : (int32_t*)workspace);
    evict_length_kernel<<<(a.ns + 127) / 128, 128, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvmem
