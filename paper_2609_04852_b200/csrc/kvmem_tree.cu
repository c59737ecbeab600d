// Attention of drafted tokens over a view (or the selected pages) and the tail of tokens behind it, and the weights it
// leaves on the view:   out_i = sum_t p_it v_t,  p_it = exp(x_it - lse_i),  x_it = scale q_i . k_t,
//                       mass_t = decay mass_t + sum_i p_it.
// A warp per query row walks the tokens 32 at a time: a lane takes one token's logit, the maximum and the sum run along
// (online softmax, fp32), then the lanes share out the 128 dimensions of the values.  The weights are a second pass once
// the log-sum-exp is known, a thread per token.
#include <math.h>

#include <algorithm>

#include "kvmem_internal.cuh"

namespace kvmem {

constexpr int kTreeD = 128;

struct TreeSpan {
    int n_view, n_tail, n_q;      // view tokens, committed tail tokens, drafted tokens of the session
};

__device__ __forceinline__ TreeSpan tree_span(const TreeArgs& a, int s, bool report) {
    TreeSpan t;
    t.n_view = (int)min((long long)max(a.n_sel[s], 0) * a.B, (long long)a.cap);
    t.n_q = a.n_q ? min(max(a.n_q[s], 0), a.M) : a.M;
    t.n_tail = 0;
    if (a.tail_k) {
        const int n = a.n_tail[s];
        t.n_tail = min(max(n, 0), a.tail_cap - t.n_q);
        if (report && t.n_tail != n) atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE);
    }
    return t;
}

// row of 128 elements of token t (view tokens first, then the tail) of KV head lg
__device__ __forceinline__ size_t view_row(const TreeArgs& a, int s, int lg, int t) {
    return (((size_t)s * a.L * a.G + lg) * a.cap + t) * kTreeD;
}
__device__ __forceinline__ size_t tail_row(const TreeArgs& a, int s, int lg, int t) {
    return (((size_t)s * a.tail_cap + t) * a.L * a.G + lg) * kTreeD;
}
__device__ __forceinline__ size_t page_row(const TreeArgs& a, int s, int lg, int t, bool value) {
    const int id = a.sel_ids[(size_t)s * a.sel_stride + t / a.B];
    int pg = -1;
    if (id >= 0 && id < a.nblocks_dev[a.session_first + s]) pg = a.tables[(size_t)(a.session_first + s) * a.max_bps + id];
    if (pg < 0 || pg >= a.max_blocks) { atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE); pg = 0; }
    return ((((size_t)pg * 2 + (value ? 1 : 0)) * a.L * a.G + lg) * a.B + t % a.B) * kTreeD;
}

__global__ void __launch_bounds__(128) tree_rows_kernel(TreeArgs a) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row = blockIdx.x * 4 + warp, lg = blockIdx.y, s = blockIdx.z;
    const TreeSpan sp = tree_span(a, s, threadIdx.x == 0);
    __shared__ float qs[4][kTreeD];
    const int m = row / a.r;
    if (row >= a.rows || m >= sp.n_q) return;
    const size_t orow = (((size_t)s * a.M + m) * a.L + lg / a.G) * a.H + (size_t)(lg % a.G) * a.r + row % a.r;
    for (int d = lane; d < kTreeD; d += 32) qs[warp][d] = __bfloat162float(a.q[orow * kTreeD + d]);
    __syncwarp();
    const unsigned long long bits = a.mask ? a.mask[(size_t)s * a.M + m] : (m >= 63 ? ~0ull : (2ull << m) - 1);
    const int end = sp.n_view + (a.tail_k ? sp.n_tail + sp.n_q : 0);
    float top = -INFINITY, z = 0.0f, o[4] = {};
    for (int t0 = 0; t0 < end; t0 += 32) {
        const int t = t0 + lane, j = t - sp.n_view - sp.n_tail;
        const bool sees = t < end && (j < 0 || ((bits >> j) & 1));
        const __nv_bfloat16 *kr = nullptr, *vr = nullptr;
        if (sees) {
            if (t >= sp.n_view) { const size_t at = tail_row(a, s, lg, t - sp.n_view); kr = a.tail_k + at; vr = a.tail_v + at; }
            else if (a.view_k) { const size_t at = view_row(a, s, lg, t); kr = a.view_k + at; vr = a.view_v + at; }
            else { kr = a.pages + page_row(a, s, lg, t, false); vr = a.pages + page_row(a, s, lg, t, true); }
        }
        float x = -INFINITY;
        if (sees) {
            x = 0.0f;
            for (int d = 0; d < kTreeD; ++d) x += qs[warp][d] * __bfloat162float(kr[d]);
            x *= a.scale;
        }
        float mx = x;
        for (int w = 16; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float nt = fmaxf(top, mx), ref = nt > -INFINITY ? nt : 0.0f;
        const float corr = expf(top - ref), p = expf(x - ref);
        float sum = p;
        for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        z = z * corr + sum;
        top = nt;
        for (int i = 0; i < 4; ++i) o[i] *= corr;
        for (int u = 0; u < 32; ++u) {
            const float pu = __shfl_sync(0xffffffffu, p, u);
            const __nv_bfloat16* vu = (const __nv_bfloat16*)__shfl_sync(0xffffffffu, (unsigned long long)vr, u);
            if (!vu) continue;                    // not visible: its value is not touched
            for (int i = 0; i < 4; ++i) o[i] += pu * __bfloat162float(vu[lane + 32 * i]);
        }
    }
    for (int i = 0; i < 4; ++i) a.out[orow * kTreeD + lane + 32 * i] = __float2bfloat16(z == 0.0f ? 0.0f : o[i] / z);
    if (lane == 0) a.lse[orow] = z == 0.0f ? -INFINITY : top + logf(z);
}

__global__ void __launch_bounds__(128) tree_mass_kernel(TreeArgs a) {
    const int t = blockIdx.x * 128 + threadIdx.x, lg = blockIdx.y, s = blockIdx.z;
    const TreeSpan sp = tree_span(a, s, false);
    if (t >= sp.n_view) return;
    const __nv_bfloat16* kr = a.view_k + view_row(a, s, lg, t);
    float w = 0.0f;
    for (int row = 0; row < sp.n_q * a.r; ++row) {
        const size_t orow = (((size_t)s * a.M + row / a.r) * a.L + lg / a.G) * a.H + (size_t)(lg % a.G) * a.r + row % a.r;
        float x = 0.0f;
        for (int d = 0; d < kTreeD; ++d) x += __bfloat162float(a.q[orow * kTreeD + d]) * __bfloat162float(kr[d]);
        w += expf(x * a.scale - a.lse[orow]);
    }
    float* mp = a.mass + ((size_t)s * a.L * a.G + lg) * a.cap + t;
    *mp = a.decay * *mp + w;
}

size_t tree_workspace_bytes(const kvmem_pool_config_t& c, int n_sessions, int n_q_tokens, int mass_cap_tokens) {
    (void)c; (void)n_sessions; (void)n_q_tokens; (void)mass_cap_tokens;
    return 256;
}

cudaError_t launch_tree(const kvmem_pool& p, const TreeArgs& a, void* workspace, cudaStream_t st) {
    (void)p; (void)workspace;
    tree_rows_kernel<<<dim3((a.rows + 3) / 4, a.L * a.G, a.ns), 128, 0, st>>>(a);
    if (a.mass) tree_mass_kernel<<<dim3((a.cap + 127) / 128, a.L * a.G, a.ns), 128, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvmem
