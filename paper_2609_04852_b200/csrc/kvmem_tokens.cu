// New tokens on their way into the cache: rotation from the model's rotary form, rows of the tail and of reserved pages, and the
// step that makes whole reserved blocks part of the repository.
//
// Rotary forms.  Every pass of this library rotates pairs (i, i + d/2) by the angles of a table row.  A model that pairs
// (2i, 2i + 1), or rotates only the first rotary_dim dims, is the same thing after a permutation of the dims, with angle 0 where
// nothing turns: pair p goes to (p, d/2 + p), the dims that pass go behind the pairs of either half.  q . k and the Mean-K score do
// not change under a permutation that queries and keys share, so only the way in knows of it ("pool's order").
//
// A thread takes 8 pairs of one vector: two 128-bit loads, the 8 (cos, sin) of the token, two 128-bit stores.  The head's dims lie
// in three orders; in each the 8 + 8 elements are two runs of 8, or one of 16 to be taken apart (interleaved pairs).
// Everything here moves bytes: bound by HBM where there are many tokens, by one launch where there are few.
//
// A thread takes one vector where all threads are resident together anyway (the shortest way through: 2.1 us instead of 2.8 with four
// vectors for 8 tokens of 40 heads, 2.5 instead of 3.8 for an append of 8 tokens with 48 heads), and several beyond, whose loads are then in
// flight together behind one table row: rotation four (24,576 tokens of 40 heads 80 us, 89 with two),
// append three (16,383 tokens with 48 heads 80 us, 83 with two, 82 with four, 101 with six).  Issue slots count beside the bytes (56 %
// busy at 65 % of HBM's cycles): indices are divided by products, the products of a rotation taken two at a time (append 90 -> 80 us).
#include <algorithm>

#include "kvmem_internal.cuh"
#include "kvmem_ptx.cuh"
#include "kvmem_t5.cuh"

namespace kvmem {

// ---- table of a rotary form -------------------------------------------------------------------------------------------------
// Angles in 64 bits, one rounding of cos and sin to fp32; one thread per entry.  A frequency of 0 gives (1, 0) exactly.
__global__ void __launch_bounds__(256)
rope_table_kernel(float2* __restrict__ rope, int half, long long entries, const __grid_constant__ RopeFrequencies f) {
    const long long e = blockIdx.x * 256ll + threadIdx.x;
    if (e >= entries) return;
    double s, c;
    sincos((double)(e / half) * f.f[e % half], &s, &c);
    rope[e] = make_float2((float)c, (float)s);
}

cudaError_t launch_rope_table(const kvmem_pool& p, const RopeFrequencies& f, cudaStream_t st) {
    const int half = p.geo.d / 2;
    const long long entries = (long long)p.cfg.rope_max_positions * half;
    rope_table_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, st>>>(p.rope_dev, half, entries, f);
    return cudaGetLastError();
}

// ---- the dims of a head ------------------------------------------------------------------------------------------------------

// where the 8 + 8 elements of chunk c lie in a vector; woven: 16 elements from lo on, pair by pair
struct Place {
    int lo, hi;
    bool woven;
};
__device__ __forceinline__ Place place_of(const RopeForm& f, bool pool_order, int c, int d) {
    if (pool_order) return {8 * c, d / 2 + 8 * c, false};
    if (c >= f.chunks) return {f.rotary + 8 * (c - f.chunks), f.rotary + (d - f.rotary) / 2 + 8 * (c - f.chunks), false};
    return f.interleaved ? Place{16 * c, 16 * c + 8, true} : Place{8 * c, f.rotary / 2 + 8 * c, false};
}

// two runs of pairs (a0 b0 a1 b1 ...) to firsts and seconds, and back
__device__ __forceinline__ void unweave(uint4& lo, uint4& hi) {
    const uint4 x = lo, y = hi;
    lo = make_uint4(__byte_perm(x.x, x.y, 0x5410), __byte_perm(x.z, x.w, 0x5410), __byte_perm(y.x, y.y, 0x5410), __byte_perm(y.z, y.w, 0x5410));
    hi = make_uint4(__byte_perm(x.x, x.y, 0x7632), __byte_perm(x.z, x.w, 0x7632), __byte_perm(y.x, y.y, 0x7632), __byte_perm(y.z, y.w, 0x7632));
}
__device__ __forceinline__ void weave(uint4& lo, uint4& hi) {
    const uint4 x = lo, y = hi;
    lo = make_uint4(__byte_perm(x.x, y.x, 0x5410), __byte_perm(x.x, y.x, 0x7632), __byte_perm(x.y, y.y, 0x5410), __byte_perm(x.y, y.y, 0x7632));
    hi = make_uint4(__byte_perm(x.z, y.z, 0x5410), __byte_perm(x.z, y.z, 0x7632), __byte_perm(x.w, y.w, 0x5410), __byte_perm(x.w, y.w, 0x7632));
}

// a chunk's angles, two pairs to a register pair
struct Angles { uint64_t c[4], s[4]; };
__device__ __forceinline__ Angles angles_at(const float2* cs, float sgn) {
    Angles t;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(cs) + w);
        t.c[w] = f2::pk(v.x, v.z);
        t.s[w] = f2::pk(sgn * v.y, sgn * v.w);
    }
    return t;
}

// 8 pairs turned: a c - b s and b c + a s, products and sums each rounded to fp32, then the amplitude's product where there is one, one
// rounding to bf16.  Products two at a time; the sums are scalar, since packed ones are contracted with the products before them.
template <bool AMPLITUDE>
__device__ __forceinline__ void turn8(uint4& lo, uint4& hi, const Angles& t, float amplitude) {
    uint32_t* l = reinterpret_cast<uint32_t*>(&lo);
    uint32_t* h = reinterpret_cast<uint32_t*>(&hi);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint64_t a = f2::pk(l[w] << 16, l[w] & 0xffff0000u), b = f2::pk(h[w] << 16, h[w] & 0xffff0000u);
        float ac0, ac1, bs0, bs1, bc0, bc1, as0, as1;
        f2::unpk(f2::mul(a, t.c[w]), ac0, ac1);
        f2::unpk(f2::mul(b, t.s[w]), bs0, bs1);
        f2::unpk(f2::mul(b, t.c[w]), bc0, bc1);
        f2::unpk(f2::mul(a, t.s[w]), as0, as1);
        float x0 = __fsub_rn(ac0, bs0), x1 = __fsub_rn(ac1, bs1), y0 = __fadd_rn(bc0, as0), y1 = __fadd_rn(bc1, as1);
        if (AMPLITUDE) { x0 = __fmul_rn(x0, amplitude); x1 = __fmul_rn(x1, amplitude); y0 = __fmul_rn(y0, amplitude); y1 = __fmul_rn(y1, amplitude); }
        l[w] = ptx::pack_bf16x2(x0, x1);
        h[w] = ptx::pack_bf16x2(y0, y1);
    }
}
__device__ __forceinline__ void turn8(uint4& lo, uint4& hi, const Angles& t, float amplitude) {
    if (amplitude != 1.0f) turn8<true>(lo, hi, t, amplitude); else turn8<false>(lo, hi, t, 1.0f);
}

__device__ __forceinline__ uint4 ld16(const __nv_bfloat16* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void st16(__nv_bfloat16* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }

// ---- rotation ----------------------------------------------------------------------------------------------------------------

// One thread: chunk c of PER vectors of one row, so that a table row is fetched once for them and their loads are in flight together.
constexpr int kTokensThreads = 128;                            // (256: 83 us instead of 80.5 for 24,576 tokens, 10.6 instead of 9.7 for 2,048)
constexpr long long kTokensFew = (long long)kSMs * 1024;      // threads that are resident together at any register count here
template <int PER>
__global__ void __launch_bounds__(kTokensThreads)
rope_apply_kernel(const __grid_constant__ RopeApplyArgs a) {
    pdl_wait();
    pdl_trigger();
    const unsigned e = blockIdx.x * (unsigned)kTokensThreads + threadIdx.x;
    const unsigned eg = a.chunks.of(e), c = a.chunks.rest(e, eg), row = a.groups.of(eg), g = a.groups.rest(eg, row);
    if (row >= (unsigned)a.n_rows) return;
    const bool turns = (int)c < a.form.chunks;
    const int pos = a.positions[row];
    if (pos < 0 || pos >= a.rope_positions) { atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE); return; }
    const Place in = place_of(a.form, a.x_pool, (int)c, a.d), out = place_of(a.form, a.y_pool, (int)c, a.d);
    const __nv_bfloat16* x = a.x + (long long)row * a.x_row + (long long)g * a.x_vec;
    __nv_bfloat16* y = a.y + (long long)row * a.y_row + (long long)g * a.y_vec;
    const long long x_step = (long long)a.groups.d * a.x_vec, y_step = (long long)a.groups.d * a.y_vec;
    uint4 lo[PER], hi[PER];
    Angles t;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if ((int)(g + i * a.groups.d) < a.n_vec) {
            // (plain loads: y may be x)
            lo[i] = *reinterpret_cast<const uint4*>(x + i * x_step + in.lo);
            hi[i] = *reinterpret_cast<const uint4*>(x + i * x_step + in.hi);
        }
    if (turns) t = angles_at(a.rope + (size_t)pos * (a.d / 2) + 8 * c, a.sgn);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if ((int)(g + i * a.groups.d) < a.n_vec) {
            if (turns) {
                if (in.woven) unweave(lo[i], hi[i]);
                turn8(lo[i], hi[i], t, a.amplitude);
                if (out.woven) weave(lo[i], hi[i]);
            }
            st16(y + i * y_step + out.lo, lo[i]);
            st16(y + i * y_step + out.hi, hi[i]);
        }
}

template <int PER>
static cudaError_t rope_apply(const kvmem_pool& p, RopeApplyArgs a, long long n_rows, cudaStream_t st) {
    a.chunks = Divisor(p.geo.d / 16);
    a.groups = Divisor((a.n_vec + PER - 1) / PER);
    const long long per_row = (long long)a.chunks.d * a.groups.d, most = std::max<long long>(1, (1ll << 30) / per_row);
    for (long long r0 = 0; r0 < n_rows; r0 += most) {
        a.n_rows = (int)std::min(most, n_rows - r0);
        const cudaError_t e = launch_pdl(rope_apply_kernel<PER>, dim3((unsigned)((a.n_rows * per_row + kTokensThreads - 1) / kTokensThreads)), dim3(kTokensThreads), 0, st, a);
        if (e != cudaSuccess) return e;
        a.x += a.n_rows * a.x_row;
        a.y += a.n_rows * a.y_row;
        a.positions += a.n_rows;
    }
    return cudaSuccess;
}

cudaError_t launch_rope_apply(const kvmem_pool& p, const RopeApplyArgs& a, long long n_rows, cudaStream_t st) {
    const bool few = n_rows <= kTokensFew / ((long long)a.n_vec * (p.geo.d / 16));
    return few ? rope_apply<1>(p, a, n_rows, st) : rope_apply<4>(p, a, n_rows, st);
}

// ---- append ------------------------------------------------------------------------------------------------------------------

// One thread: chunk c of PER vectors of one new token, a vector being a query, key or value head of a layer.  Vectors are numbered
// [layer][query heads | key heads | value heads].  What a thread needs comes in two rounds of loads: counts, lengths and its vectors,
// then the table row and the page.
template <int PER>
__global__ void __launch_bounds__(kTokensThreads)
append_tokens_kernel(const __grid_constant__ AppendTokensArgs a) {
    pdl_wait();
    pdl_trigger();
    const unsigned e = blockIdx.x * (unsigned)kTokensThreads + threadIdx.x;
    const unsigned eg = a.chunks.of(e), c = a.chunks.rest(e, eg), token = a.groups.of(eg), g = a.groups.rest(eg, token);
    const unsigned s1 = a.tokens.of(token), i = a.tokens.rest(token, s1), s = s1 + (unsigned)a.s0;
    if (s >= (unsigned)a.ns) return;
    const int given_new = a.n_new ? a.n_new[s] : a.M, given = a.tail_n[s];
    const int n_sel = a.rope && a.n_sel ? a.n_sel[s] : 0, at = a.rope && a.positions ? a.positions[(size_t)s * a.M + i] : 0;
    const int blocks = a.pages ? a.nblocks_dev[a.session_first + s] : 0;
    const bool turns = (int)c < a.form.chunks;
    const Place in = place_of(a.form, a.rope == nullptr, (int)c, a.d);
    const int lo_at = 8 * (int)c, hi_at = a.d / 2 + 8 * (int)c;
    uint4 lo[PER], hi[PER];
    int kind[PER], l[PER], h[PER];                       // 0 query, 1 key, 2 value, -1 none; layer; head
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const unsigned v = g + u * a.groups.d;
        kind[u] = -1;
        if ((int)v < a.n_vec) {
            l[u] = (int)a.per_layer.of(v);
            h[u] = (int)a.per_layer.rest(v, l[u]);
            kind[u] = 0;
            if (h[u] >= a.Hq) { h[u] -= a.Hq; kind[u] = 1; }
            if (kind[u] == 1 && h[u] >= a.G) { h[u] -= a.G; kind[u] = 2; }
            const TokenRows& t = kind[u] == 0 ? a.q : kind[u] == 1 ? a.k : a.v;
            const __nv_bfloat16* src = t.data + (long long)s * t.session + (long long)i * t.token + (l[u] * t.layer + h[u] * t.head);
            lo[u] = ld16(src + (kind[u] == 2 ? lo_at : in.lo));
            hi[u] = ld16(src + (kind[u] == 2 ? hi_at : in.hi));
        }
    }
    const int n_new = min(max(given_new, 0), a.M);
    if ((int)i >= n_new) return;
    const int n_tail = min(max(given, 0), a.tail_cap - n_new), row = n_tail + (int)i;
    bool ok = n_tail == given;
    Angles t;
    if (a.rope) {
        const long long pos = a.positions ? at : (long long)a.first_position + (long long)max(n_sel, 0) * a.B + row;
        if (pos < 0 || pos >= a.rope_positions) { atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE); return; }
        if (turns) t = angles_at(a.rope + (size_t)pos * (a.d / 2) + 8 * c, 1.0f);
    }
    __nv_bfloat16* page = nullptr;
    if (a.pages) {
        const int rb = (int)a.block.of(row), b = blocks + rb;
        const int pg = b < a.max_bps ? a.tables[(size_t)(a.session_first + s) * a.max_bps + b] : -1;
        if (pg >= 0 && pg < a.max_blocks) page = a.pages + (size_t)pg * a.page_elems + (int)a.block.rest(row, rb) * a.d;
        else ok = false;
    }
    if (!ok) atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE);
    // a token's vectors lie within 2^31 elements of one another, in every result
    __nv_bfloat16 *const q_out = a.q_out + ((size_t)s * a.M + i) * (size_t)(a.L * a.Hq * a.d);
    const size_t tail_row = ((size_t)s * a.tail_cap + row) * (size_t)(a.L * a.G * a.d);
    const int tile = a.B * a.d;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        if (kind[u] < 0) continue;
        if (kind[u] < 2 && turns && in.woven) unweave(lo[u], hi[u]);
        const int place = l[u] * a.G + h[u];                               // of a key or value
        if (kind[u] > 0 && page) {
            __nv_bfloat16* dst = page + (place + (kind[u] == 2 ? a.L * a.G : 0)) * (size_t)tile;
            st16(dst + lo_at, lo[u]);
            st16(dst + hi_at, hi[u]);
        }
        if (kind[u] < 2 && turns) turn8(lo[u], hi[u], t, kind[u] == 0 ? a.q_amplitude : 1.0f);
        __nv_bfloat16* dst = kind[u] == 0 ? q_out + (l[u] * a.Hq + h[u]) * a.d : (kind[u] == 1 ? a.tail_k : a.tail_v) + tail_row + place * a.d;
        st16(dst + lo_at, lo[u]);
        st16(dst + hi_at, hi[u]);
    }
}

template <int PER>
static cudaError_t append_tokens(AppendTokensArgs a, cudaStream_t st) {
    a.groups = Divisor((a.n_vec + PER - 1) / PER);
    // whole sessions per launch, as far as their threads stay below 2^30 (the caller keeps one session below that)
    const long long per_session = (long long)a.M * a.chunks.d * a.groups.d;
    const int most = (int)std::max<long long>(1, (1ll << 30) / per_session), all = a.ns;
    for (int s0 = 0; s0 < all; s0 += most) {
        a.s0 = s0;
        a.ns = std::min(all, s0 + most);
        const long long blocks = ((a.ns - s0) * per_session + kTokensThreads - 1) / kTokensThreads;
        const cudaError_t e = launch_pdl(append_tokens_kernel<PER>, dim3((unsigned)blocks), dim3(kTokensThreads), 0, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_append_tokens(const kvmem_pool& p, AppendTokensArgs a, cudaStream_t st) {
    a.chunks = Divisor(p.geo.d / 16);
    a.n_vec = a.L * (a.Hq + 2 * a.G);
    a.tokens = Divisor(a.M);
    a.per_layer = Divisor(a.Hq + 2 * a.G);
    a.block = Divisor(a.B);
    const bool few = (long long)a.ns * a.M <= kTokensFew / ((long long)a.n_vec * a.chunks.d);
    return few ? append_tokens<1>(a, st) : append_tokens<3>(a, st);
}

bool append_tokens_fits(const kvmem_pool_config_t& c, int n_q_tokens) {
    const long long vectors = (long long)c.n_layers * (c.n_q_heads + 2ll * c.n_kv_heads);
    return vectors * c.head_dim < (1ll << 31) && (double)n_q_tokens * (c.head_dim / 16) * (double)vectors < (double)(1ll << 31);
}

// ---- commit ------------------------------------------------------------------------------------------------------------------
// Three launches once in a block's worth of tokens, built for the bits of append_kernel and a tail moved in place.  Bound by
// latency, far from the bytes' time: the sum over a block's tokens is a chain of additions in token order, and a tail goes down in runs of the
// committed tokens, one behind the other.  Cold, us on the device (floor by bytes): 8 sessions of a block and a token 40 (0.2), a chunk of
// 32 blocks 44 (0.7), a prompt of 256 blocks 42 (5.2), one block out of a tail of 2,048 tokens 167 (2.5; 31 runs), 16 blocks out of it 101 (1.6).

// Index rows of blocks whose raw keys lie in pages already: the fp32 sum in token order, one product, one rounding of append_kernel,
// a thread per dim.  Grid: (block of the session, layer and KV head, session).
__global__ void __launch_bounds__(128)
commit_index_kernel(const __grid_constant__ CommitArgs a) {
    const CommitSession cs = a.s[blockIdx.z];
    const int b = cs.have + (int)blockIdx.x, lg = blockIdx.y;
    if ((int)blockIdx.x >= cs.n) return;
    const int pg = a.tables[(size_t)cs.session * a.max_bps + b];
    if (pg < 0 || pg >= a.max_blocks) { if (threadIdx.x == 0) atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE); return; }
    const __nv_bfloat16* k = a.pages + (size_t)pg * a.page_elems + (size_t)lg * a.B * a.d;
    __nv_bfloat16* row = a.index + (size_t)cs.session * a.index_elems + ((size_t)lg * a.max_bps + b) * a.d;
    const float inv = 1.0f / (float)a.B;
    for (int x = threadIdx.x; x < a.d; x += 128) {
        float acc = 0.0f;
#pragma unroll 16
        for (int t = 0; t < a.B; ++t) acc = __fadd_rn(acc, __bfloat162float(k[(size_t)t * a.d + x]));
        row[x] = __float2bfloat16_rn(__fmul_rn(acc, inv));
    }
}

// The tail's rows behind the committed blocks move to its front: n B rows down, in runs of at most that many, so that a run's reads
// and writes never meet; 16 bytes a thread.  Grid: (16-byte columns of a token row / 32, K | V, session).
__global__ void __launch_bounds__(256)
commit_tail_kernel(const __grid_constant__ CommitArgs a) {
    const CommitSession cs = a.s[blockIdx.z];
    const int down = cs.n * a.B, n = min(a.tail_n[cs.slot], a.tail_cap), left = n - down;
    if (left <= 0) return;                              // fewer than the blocks hold: commit_counts_kernel reports it
    const size_t width = (size_t)a.L * a.G * a.d / 8;   // 16-byte columns
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
    uint4* t = reinterpret_cast<uint4*>(blockIdx.y ? a.tail_v : a.tail_k) + (size_t)cs.slot * a.tail_cap * width + col;
    for (int r0 = 0; r0 < left; r0 += down) {
        const int end = min(left, r0 + down);
        if ((size_t)col < width)
            for (int r = r0 + lane; r < end; r += 8) t[(size_t)r * width] = t[(size_t)(r + down) * width];
        __syncthreads();
    }
}

__global__ void commit_counts_kernel(const __grid_constant__ CommitArgs a) {
    const CommitSession cs = a.s[threadIdx.x];
    if ((int)threadIdx.x >= a.ns) return;
    a.nblocks[cs.session] = cs.have + cs.n;
    if (a.tail_n) {
        const int n = a.tail_n[cs.slot], left = min(n, a.tail_cap) - cs.n * a.B;
        if (left < 0 || n > a.tail_cap) atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE);
        a.tail_n[cs.slot] = max(left, 0);
    }
}

cudaError_t launch_commit(const CommitArgs& a, cudaStream_t st) {
    int most = 0;
    for (int i = 0; i < a.ns; ++i) most = std::max(most, a.s[i].n);
    commit_index_kernel<<<dim3((unsigned)most, (unsigned)(a.L * a.G), (unsigned)a.ns), 128, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (a.tail_n) {
        const unsigned cols = (unsigned)(((size_t)a.L * a.G * a.d / 8 + 31) / 32);
        commit_tail_kernel<<<dim3(cols, 2, (unsigned)a.ns), 256, 0, st>>>(a);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    commit_counts_kernel<<<1, kCommitSessions, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvmem
