// Attention of a prompt chunk over a view and the tail of tokens behind it, the chunk's own tokens among them:
//   out_i = sum_t p_it v_t,  p_it = exp(x_it - lse_i),  x_it = scale q_i . k_t  over the view's tokens, the committed tail tokens and
//   the chunk tokens 0 .. i.
//
// The arithmetic is the tensor pipe's: 4 d flops per query row and token against 2 d bytes of key and value that many rows share.
// A CTA works on two row tiles of 128 query rows at a time (whole tokens times the r query heads of a KV head), a slot each:
//     S = Q K^T    tcgen05.mma, both operands in shared memory, 128 x 128 fp32 accumulators in tensor memory
//     P = exp2(S scale log2e - ref)     four warps a slot, a thread per row: no exchange between threads
//     O += P V     tcgen05.mma, P as bf16 in tensor memory (over S), V from shared memory
// so that one slot's products run while the other's weights are computed.  S, P and O of the two slots fill tensor memory.  One
// thread fetches Q, K and V tiles with TMA (128-byte swizzle), one thread issues the MMAs: those of one thread run in order, so a
// slot's next S is issued right behind the product that reads its P, in whose place it goes.
//
// ref is the largest logit of the first tokens a row sees.  It moves only when the row's weights sum to more than 2^15, to that sum's
// logarithm or to the half tile's largest logit, whichever is more: O is then rescaled in tensor memory and the half's weights are
// computed again.  Until then they may be that large, which costs neither fp32 nor bf16 any precision, and no tile needs the maximum of
// its logits.  O stays below 2^15 times the largest value however long the view is, so values up to 2^112 do not overflow it.
//
// Work: an item is (session, KV head, group of two row tiles); its tiles are those of the view and of the tail up to the group's last
// token.  All items' tiles lie on one line (with a lead for what starting and ending an item costs), cut into equal parts, one for each
// CTA (one per SM): chunks over views of any lengths keep all SMs busy to the end, and the causal part's short and long items need
// no other balance.  An item that a cut falls into is left as partial sums, joined in line order by prefill_merge_kernel: the
// result depends on the sizes alone, not on timing.  A part leaves at most two of them (its first and its last), so the workspace
// does not grow with the call.
// Where the keys and values of all KV heads are more than L2 holds, the line is cut into several parts for each CTA, the c-th of n from
// c on in steps of n: all CTAs then work on a few heads at a time and find their tiles in L2 after the first.  (In one sweep over
// eight heads of 33 MB the CTAs are spread over all of them and read every tile from HBM: 2,048 tokens over 65,536 take 2,200 us at
// 1,342 MHz under the power limit; in four sweeps 1,937 us at 1,567 MHz.)
//
// Tokens that a row does not see: their logits are replaced before they are used, values behind the last token are cleared in shared
// memory before the second product (0 x NaN), and so are values that are not finite of chunk tokens that only some rows see; the
// rows that do see them get them at the end.  Two warps of their own look at those values while the logits are on their way (by the row
// warps: 159 us instead of 155 for a chunk of 4,096 alone).
//
// What bounds it: under a long view the power limit (960 W at 1,567 MHz) and the chain S -> weights -> O of each slot: 3,300 cycles per
// 128 tokens of 256 rows, where the products alone take 2,048 by their rate, 2,724 with operands that lie in shared memory already, some
// 2,900 with the tiles' loads beside them.  2,048 tokens of 32 heads on 8 over 65,536: 1,705 us before the power limit bites, 1,915 behind
// it (1,310 and 1,168 TFLOP/s).  Short calls: 2 us of plan, 2.6 to the first tile, 2 us for a CTA's every further item, 5 of joining.
// Measured and dropped: two threads a row (16 row warps; 221 us instead of 197 for 4,096 alone), an MMA thread a slot (170, 163), S in two
// halves of 64 tokens (211, 195), a part of the exponentials by a polynomial (an eighth: 174, 155), fewer tokens in the last product of
// a causal item (171, 162: what the MMA thread does between two products costs more).
#include <cudaTypedefs.h>
#include <math.h>

#include <algorithm>

#include "kvmem_internal.cuh"
#include "kvmem_ptx.cuh"
#include "kvmem_t5.cuh"

namespace kvmem {

constexpr int kPreD = 128;
constexpr int kPreTile = 128;                    // tokens per tile
constexpr int kPreRows = 128;                    // rows per slot: TMEM lanes
constexpr int kPreHalf = 128 * 128;              // bytes of one 64-dim half of a 128-row operand tile
constexpr int kPreSlot = 2 * kPreHalf;           // a K, V or Q tile
constexpr int kPreRing = 4;                      // K and V tiles in turn
constexpr int kPreStage = 4096;                  // bytes of a row warp's staging for stores
constexpr int kPreThreads = 384;                 // eight row warps, TMA warp, MMA warp, two for values that rows do not see
constexpr int kPreTmaWarp = 8, kPreMmaWarp = 9;
// Registers a thread: the launch gives 168, the row warps take 208 and the others keep 88.  (Without: a row's 128 logits do not fit, and a
// spill is slow here, where shared memory leaves the L1 no room for it: 220 us instead of 206 for a chunk of 4,096 alone.  With 80 for
// the others 161 instead of 159.)
#define PRE_ROW_REGS "208"
#define PRE_OTHER_REGS "88"
static_assert(256 * 208 + 128 * 88 <= kPreThreads * 168, "the registers that the row warps take are those the others give");
constexpr int kPreLead = 3;                      // units on the line for an item's start and end: what they cost a CTA, in tiles (1: 170 and 243 us,
                                                 // 5: 159 and 212, instead of 155 and 214 for a chunk of 4,096 alone and three ragged sessions)
constexpr float kPreLimit = 32768.0f;            // a row's weights may sum to this before their reference moves (2^12 instead: 2,240 us against 1,959
                                                 // for 2,048 tokens over 65,536, 233 against 219 for three ragged sessions; 2^17 and 2^20 as 2^15)
constexpr int kPreParts = 4;                     // parts of the line a CTA can have
constexpr int kPreBudget = 1024;                 // tiles of keys and values (64 KiB each) that a sweep of all CTAs may hold in L2
constexpr int kPrePartUnits = 64;                // least units of a part, when there is more than one
constexpr uint32_t kPreIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (16u << 17) | (8u << 24);   // bf16 x bf16 -> fp32, 128 x 128
constexpr uint32_t kPreIdescO = kPreIdescS | (1u << 16);                                         // B with dims contiguous (V as it lies)
constexpr uint32_t kPreVStep = (uint32_t)kPreHalf >> 4;       // leading offset of V's descriptor: from dims 0..63 to 64..127
constexpr int kPreMostUnits = 1 << 30;

struct PreRecord { int s, lg, rg, last; };       // an item, and the part its last share lies in; s < 0: none

struct PreWork {
    PrefillArgs a;
    int tpt;                                     // tokens per row tile
    int log_group;                               // log2 of the tokens of a group, where they are a power of two; else -1
    float* part_o;                               // [2 parts][slot][dims / 4][128 rows][4]
    float2* part_ml;                             // [2 parts][256]: (reference, sum of weights), log2 domain
    PreRecord* rec;                              // [2 parts]: what shares 2c (begun in an earlier part) and 2c + 1 (goes on in the next) hold
    int* nf;                                     // [2 parts]: whether values that are not finite were cleared
    int* n_parts;                                // parts of the line in all
};

struct PreSpan {
    int n_view, n_tail, n_q, view_tiles, groups;
};

__device__ __forceinline__ PreSpan pre_span(const PrefillArgs& a, int tpt, int s, bool report) {
    PreSpan t;
    t.n_view = (int)min((long long)max(a.n_sel[s], 0) * a.B, (long long)a.cap);
    t.n_q = a.n_q ? min(max(a.n_q[s], 0), a.M) : a.M;
    t.n_tail = 0;
    if (a.tail_k) {
        const int n = a.n_tail[s];
        t.n_tail = min(max(n, 0), a.tail_cap - t.n_q);
        if (report && t.n_tail != n) atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE);
    }
    t.view_tiles = (t.n_view + kPreTile - 1) / kPreTile;
    t.groups = (t.n_q + 2 * tpt - 1) / (2 * tpt);
    return t;
}

// tail tokens that the last row of group rg sees, in tiles
__device__ __forceinline__ int pre_tail_tiles(const PrefillArgs& a, const PreSpan& sp, int tpt, int rg) {
    return a.tail_k ? (sp.n_tail + min((rg + 1) * 2 * tpt, sp.n_q) + kPreTile - 1) / kPreTile : 0;
}

// sum over i < n of floor((step i + from) / 128): whole parts of step and from taken out, then the axes of the lattice points under the line
// exchanged, as in Euclid's algorithm (a known method; Knuth, The Art of Computer Programming, 3.3.3; Graham, Knuth and Patashnik,
// Concrete Mathematics, 3.5).  In 32 bits: the sum is
// at most the line's 2^30 units, and so are the products that it is made of.
__device__ __forceinline__ uint32_t floor_sum(uint32_t n, uint32_t step, uint32_t from) {
    uint32_t m = kPreTile, sum = 0;
    while (n > 0) {
        if (step >= m) { const uint32_t k = step / m; sum += (n - 1) * n / 2 * k; step -= k * m; }
        if (from >= m) { const uint32_t k = from / m; sum += n * k; from -= k * m; }
        const uint32_t top = step * n + from;
        if (top < m) break;
        n = top / m;
        from = top - n * m;
        const uint32_t t = m;
        m = step;
        step = t;
    }
    return sum;
}

// the same where step is 2^log: without a division
__device__ __forceinline__ uint32_t floor_sum_pow2(uint32_t n, int log, uint32_t from) {
    constexpr int m = 7;                                                // log2 of 128
    if (log >= m) return ((n * (n - 1) / 2) << (log - m)) + n * (from >> m);
    const int k = m - log;                                              // floor((2^log i + from) / 128) = floor((i + from / 2^log) / 2^k)
    auto upto = [&](uint32_t x) { const uint32_t q = x >> k; return ((q * (q - 1) / 2) << k) + q * (x - (q << k)); };       // over i < x of floor(i / 2^k)
    return upto(n + (from >> log)) - upto(from >> log);
}

// units of the row groups before group rg of a KV head (rg < groups), and of a whole KV head.  An item without a tile (no view, no
// tail) has one unit beside its lead: somebody has to write its rows.
__device__ __forceinline__ int pre_before(const PreWork& w, const PreSpan& sp, int rg) {
    if (!w.a.tail_k) return rg * (max(sp.view_tiles, 1) + kPreLead);
    const uint32_t from = (uint32_t)(sp.n_tail + 2 * w.tpt + kPreTile - 1);
    return rg * (sp.view_tiles + kPreLead) + (int)(w.log_group >= 0 ? floor_sum_pow2(rg, w.log_group, from) : floor_sum(rg, 2 * w.tpt, from));
}
__device__ __forceinline__ int pre_tiles(const PrefillArgs& a, const PreSpan& sp, int tpt, int rg) { return sp.view_tiles + pre_tail_tiles(a, sp, tpt, rg); }
__device__ __forceinline__ int pre_head(const PreWork& w, const PreSpan& sp) {
    if (sp.groups == 0) return 0;
    return pre_before(w, sp, sp.groups - 1) + max(pre_tiles(w.a, sp, w.tpt, sp.groups - 1), 1) + kPreLead;
}

// where a part of the line begins and ends, and the item at its beginning: its first unit, session, KV head, row group
struct PrePart { int begin, end, from, s, lg, rg; };

// a role's walk over its CTA's shares of items
struct PreWalk {
    const PrePart* parts;           // the CTA's, in shared memory
    int part, n_parts;              // the next one, how many
    int pos, end, from;             // next unit of the line, the part's end, the item's first unit
    int s, lg, rg;                  // the item at `from`
    PreSpan sp;
    int t0, t1, tiles;              // the share: tiles [t0, t1) of the item's `tiles` (0: nothing to see)
    int cs, clg, crg, m0, rows2;    // its item; first token; whether the second row tile has any token
    int last;                       // the item's last unit
    bool more;
    __device__ __forceinline__ bool next(const PreWork& w, int LG) {
        const PrefillArgs& a = w.a;
        while (true) {
            if (pos >= end) {
                if (part >= n_parts) return false;
                const PrePart p = parts[part++];
                pos = p.begin; end = p.end; from = p.from; s = p.s; lg = p.lg; rg = p.rg;
                sp = pre_span(a, w.tpt, s, false);
            }
            while (sp.groups == 0) sp = pre_span(a, w.tpt, ++s, false);     // (a session that has units follows: pos < end)
            tiles = pre_tiles(a, sp, w.tpt, rg);
            const int some = max(tiles, 1), first = from + kPreLead, item_end = first + some;
            t0 = max(pos - first, 0);
            t1 = min(some, end - first);
            cs = s; clg = lg; crg = rg; last = item_end - 1;
            m0 = rg * 2 * w.tpt;
            rows2 = sp.n_q - m0 > w.tpt;
            n_view = sp.n_view; n_tail = sp.n_tail; n_q = sp.n_q; view_tiles = sp.view_tiles;
            pos = min(end, item_end);
            if (pos == item_end) {
                from = item_end;
                if (++rg == sp.groups) {
                    rg = 0;
                    if (++lg == LG) {
                        lg = 0;
                        if (pos < end) sp = pre_span(a, w.tpt, ++s, false);
                    }
                }
            }
            if (t0 < t1) return true;
        }
    }
    int n_view, n_tail, n_q, view_tiles;      // of the share's session
    __device__ __forceinline__ int units() const { return tiles ? t1 - t0 : 0; }
    // of the share's tile t: its first token in view or tail, its tokens, those that every row sees, whether some do not
    __device__ __forceinline__ int first_of(int t) const { return (t < view_tiles ? t : t - view_tiles) * kPreTile; }
    __device__ __forceinline__ int valid_of(int t) const { return (t < view_tiles ? n_view : n_tail + n_q) - first_of(t); }
    __device__ __forceinline__ int plain_of(int t) const { return t < view_tiles ? valid_of(t) : min(valid_of(t), n_tail + m0 + 1 - first_of(t)); }
    __device__ __forceinline__ bool cleans(int t) const { return plain_of(t) < kPreTile; }
};

struct PreShared {
    uint64_t full[kPreRing], empty[kPreRing], q_full, q_empty, s_full[2], p_full[2][2], h_full[2], o_full[2], o_empty[2], v_ask, v_clean, drained;
    PrePart parts[kPreParts];
    PreWalk walk[8];                          // of the row warps
    int n_parts, n_cta, total;                // the CTA's; CTAs that share the line, its units
    uint32_t tmem;
    int loads;                                // tiles requested so far: waits of many tiles' length look at it
    int not_finite[4];                        // by the share's number mod 4: that number + 1, where values were cleared
};
// A wait that may last as long as a share (seconds, where one head's view fills the device): given up when no tile was requested
// between two limits.
__device__ __forceinline__ bool pre_wait_long(const PreShared& sh, uint64_t* bar, uint32_t ph) {
    for (int seen = -1;;) {
        if (ptx::mbar_wait(bar, ph)) return true;
        const int now = *(const volatile int*)&sh.loads;
        if (now == seen) return false;
        seen = now;
    }
}
constexpr size_t kPreSmem = (size_t)(2 + kPreRing) * kPreSlot + 8 * kPreStage + sizeof(PreShared);
static_assert(kPreSmem <= 232448, "shared memory of a CTA");

__device__ __forceinline__ void pre_zero_row(const PrefillArgs& a, size_t orow) {
    uint4* o = reinterpret_cast<uint4*>(a.out + orow * kPreD);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = make_uint4(0u, 0u, 0u, 0u);
    a.lse[orow] = -INFINITY;
}

__global__ void __launch_bounds__(kPreThreads, 1)
prefill_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
               const __grid_constant__ CUtensorMap map_tk, const __grid_constant__ CUtensorMap map_tv, const __grid_constant__ PreWork w) {
    constexpr int RING = kPreRing;
    extern __shared__ __align__(1024) unsigned char smem_q[];          // two Q tiles, the ring, then the small things
    const PrefillArgs& a = w.a;
    unsigned char* ring = smem_q + 2 * kPreSlot;
    unsigned char* staging = ring + (size_t)RING * kPreSlot;
    PreShared& sh = *reinterpret_cast<PreShared*>(staging + 8 * kPreStage);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int LG = a.L * a.G, tpt = w.tpt;

    if (ptx::smem_u32(smem_q) & 1023u) {          // never: nothing static lies in front of the dynamic part
        if (tid == 0) atomicExch(a.status, (int)KVMEM_E_UNSUPPORTED);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < RING; ++i) { ptx::mbar_init(&sh.full[i], 1); ptx::mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sh.s_full[i], 1);
            ptx::mbar_init(&sh.p_full[i][0], 4);
            ptx::mbar_init(&sh.p_full[i][1], 4);
            ptx::mbar_init(&sh.h_full[i], 1);
            ptx::mbar_init(&sh.o_full[i], 1);
            ptx::mbar_init(&sh.o_empty[i], 4);
            sh.not_finite[i] = sh.not_finite[2 + i] = 0;
        }
        ptx::mbar_init(&sh.q_full, 1);
        ptx::mbar_init(&sh.q_empty, 1);
        ptx::mbar_init(&sh.v_ask, 1);
        ptx::mbar_init(&sh.v_clean, 2);
        ptx::mbar_init(&sh.drained, 1);
        sh.loads = 0;
        ptx::fence_mbar_init();
    }
    if (warp == kPreMmaWarp) {
        t5::tmem_alloc(&sh.tmem, 512);
        t5::tmem_relinquish();
    }
    pdl_wait();        // everything earlier in the stream is complete and visible from here on
    pdl_trigger();
    if (tid == 32 * kPreTmaWarp) {
        ptx::prefetch_tensormap(&map_q);
        ptx::prefetch_tensormap(&map_k);
        ptx::prefetch_tensormap(&map_v);
        ptx::prefetch_tensormap(&map_tk);
        ptx::prefetch_tensormap(&map_tv);
    }
    {
        // the CTA's parts of the line, and the item each starts in: a warp a part, each counting the line for itself
        const PreSpan first = lane < a.ns ? pre_span(a, tpt, lane, blockIdx.x == 0 && warp == 0) : PreSpan{};
        const int first_head = pre_head(w, first);
        int sum = first_head, held = first.groups ? pre_tiles(a, first, tpt, first.groups - 1) : 0;
        for (int s = lane + 32; s < a.ns; s += 32) {
            const PreSpan sp = pre_span(a, tpt, s, blockIdx.x == 0 && warp == 0);
            sum += pre_head(w, sp);
            held += sp.groups ? pre_tiles(a, sp, tpt, sp.groups - 1) : 0;
        }
        const int total = __reduce_add_sync(0xffffffffu, sum) * LG, n = min((int)gridDim.x, total);
        const unsigned tiles = __reduce_add_sync(0xffffffffu, held) * (unsigned)LG;
        int sweeps = (int)min((unsigned)kPreParts, (tiles + kPreBudget - 1) / kPreBudget);
        sweeps = max(1, min(sweeps, n ? total / (n * kPrePartUnits) : 1));
        const int all = n * sweeps, mine_n = (int)blockIdx.x < n ? sweeps : 0;
        // parts begin at floor(total part / all): in 32 bits, all being at most kSMs kPreParts
        const unsigned each = all ? (unsigned)total / (unsigned)all : 0u, over = (unsigned)total - each * (unsigned)all;
        for (int b = warp; b < mine_n; b += kPreThreads / 32) {
            const int part = b * n + (int)blockIdx.x;
            const int begin = (int)(each * part + over * part / (unsigned)all), end = (int)(each * (part + 1) + over * (part + 1) / (unsigned)all);
            int before = 0;
            for (int s0 = 0; s0 < a.ns; s0 += 32) {
                const int s = s0 + lane;
                PreSpan sp{};
                int head = 0;
                if (s0 == 0) { sp = first; head = first_head; }
                else if (s < a.ns) { sp = pre_span(a, tpt, s, false); head = pre_head(w, sp); }
                const int mine = head * LG;
                int incl = mine;
                if (a.ns > 1) {
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int up = __shfl_up_sync(0xffffffffu, incl, d);
                        if (lane >= d) incl += up;
                    }
                }
                const int lo = before + incl - mine;
                const unsigned here = __ballot_sync(0xffffffffu, begin >= lo && begin < lo + mine);
                if (here) {
                    // that lane's session; the last of its row groups that starts at the part's beginning or before, 32 tried at a time
                    const int from = __ffs(here) - 1;
                    const int at_s = s0 + from, lo_s = __shfl_sync(0xffffffffu, lo, from), head_s = __shfl_sync(0xffffffffu, head, from);
                    sp.n_view = __shfl_sync(0xffffffffu, sp.n_view, from); sp.n_tail = __shfl_sync(0xffffffffu, sp.n_tail, from);
                    sp.n_q = __shfl_sync(0xffffffffu, sp.n_q, from); sp.view_tiles = __shfl_sync(0xffffffffu, sp.view_tiles, from);
                    sp.groups = __shfl_sync(0xffffffffu, sp.groups, from);
                    const int lg = (begin - lo_s) / head_s, at = begin - lo_s - lg * head_s;
                    int rg = 0, units = 0;
                    for (int span = sp.groups; span > 0;) {
                        const int step = (span + 31) / 32, try_rg = rg + lane * step, u = lane * step < span ? pre_before(w, sp, try_rg) : 0;
                        const int k = 31 - __clz(__ballot_sync(0xffffffffu, lane * step < span && u <= at));
                        units = __shfl_sync(0xffffffffu, u, k);
                        rg += k * step;
                        span = step == 1 ? 0 : min(step, span - k * step);
                    }
                    if (lane == 0) sh.parts[b] = PrePart{begin, end, lo_s + lg * head_s + units, at_s, lg, rg};
                    break;
                }
                before += __shfl_sync(0xffffffffu, incl, 31);
            }
            if (lane == 0) {
                w.rec[2 * part].s = -1;
                w.rec[2 * part + 1].s = -1;
            }
        }
        if (tid == 0) {
            sh.n_parts = mine_n;
            sh.n_cta = n;
            sh.total = total;
            if (blockIdx.x == 0) *w.n_parts = all;
        }
    }
    t5::fence_before();
    __syncthreads();
    t5::fence_after();
    const uint32_t tmem = sh.tmem;
    PreWalk walk0;
    walk0.parts = sh.parts; walk0.n_parts = sh.n_parts;
    walk0.part = walk0.pos = walk0.end = 0;

    // A wait that runs out is recorded and the role goes on without waiting (and without issuing what would need it), so that
    // every role still reaches its end.
    bool ok = true;
    if (warp >= kPreTmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 " PRE_OTHER_REGS ";");
        PreWalk walk = walk0;
        if (warp == kPreTmaWarp) {
            // ------------------------------------------------ TMA: one thread
            if (t5::elect()) {
                int n = 0, seg = 0;                                       // loads of the ring, shares so far
                auto slot = [&]() {                                       // the next ring slot, free
                    const int st = n % RING;
                    if (ok && n >= RING) ok = ptx::mbar_wait(&sh.empty[st], (uint32_t)(((n / RING) & 1) ^ 1));
                    ++n;
                    return st;
                };
                while (ok && walk.next(w, LG)) {
                    const int units = walk.units();
                    if (units == 0) continue;
                    if (seg > 0) ok = ptx::mbar_wait(&sh.q_empty, (uint32_t)((seg - 1) & 1));
                    if (!ok) break;
                    const int l = walk.clg / a.G, g = walk.clg % a.G, tok0 = walk.cs * a.M + walk.m0;
                    ptx::mbar_expect_tx(&sh.q_full, (uint32_t)((walk.rows2 ? 2 : 1) * 2 * 128 * a.r * tpt));
                    for (int x = 0; x <= walk.rows2; ++x)
                        for (int h = 0; h < 2; ++h)
                            ptx::tma_load_3d(smem_q + x * kPreSlot + h * kPreHalf, &map_q, 64 * h, l * a.H + g * a.r, tok0 + x * tpt, &sh.q_full);
                    const int z_view = walk.cs * LG + walk.clg, row_tail = walk.cs * a.tail_cap;
                    for (int t = walk.t0; t < walk.t1 && ok; ++t) {
                        const bool in_view = t < walk.view_tiles;
                        const int c0 = (in_view ? t : t - walk.view_tiles) * kPreTile;
                        for (int kv = 0; kv < 2; ++kv) {
                            const int st = slot();
                            if (!ok) { --n; break; }
                            unsigned char* dst = ring + (size_t)st * kPreSlot;
                            ptx::mbar_expect_tx(&sh.full[st], kPreSlot);
                            for (int h = 0; h < 2; ++h) {
                                if (in_view) ptx::tma_load_3d(dst + h * kPreHalf, kv ? &map_v : &map_k, 64 * h, c0, z_view, &sh.full[st]);
                                else ptx::tma_load_3d(dst + h * kPreHalf, kv ? &map_tv : &map_tk, 64 * h, walk.clg, row_tail + c0, &sh.full[st]);
                            }
                        }
                        *(volatile int*)&sh.loads = n;
                    }
                    ++seg;
                }
                // the copies still in flight land before the CTA gives its shared memory back
                for (int i = max(0, n - RING); i < n; ++i) ok = ptx::mbar_wait(&sh.full[i % RING], (uint32_t)((i / RING) & 1)) && ok;
                if (seg > 0) ok = ptx::mbar_wait(&sh.q_full, (uint32_t)((seg - 1) & 1)) && ok;
                if (!ok) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
            }
        } else if (warp == kPreMmaWarp) {
            // ------------------------------------------------ MMA: one thread
            if (t5::elect()) {
                const uint32_t q_lo = t5::desc_lo(ptx::smem_u32(smem_q)), ring_lo = t5::desc_lo(ptx::smem_u32(ring));
                struct Place {                                            // ring slot and phase of the next key / value tile
                    int st;
                    uint32_t ph;
                    __device__ __forceinline__ void next() { st += 2; if (st >= RING) { st -= RING; ph ^= 1u; } }
                } kp{0, 0u}, vp{1, 0u};
                int seg = 0;
                uint32_t p_ph0 = 0, p_ph1 = 0;                            // phases of the slots' weights
                int out0 = 0, out1 = 0;                                   // shares whose sums a slot's rows have to take out
                auto logits = [&](int x) {
                    if (!ok) return;
                    t5::fence_after();
                    const uint32_t al = q_lo + (uint32_t)x * (kPreSlot >> 4), bl = ring_lo + (uint32_t)kp.st * (kPreSlot >> 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t o = (uint32_t)(i >> 2) * (kPreHalf >> 4) + (uint32_t)(i & 3) * 2u;
                        t5::mma_bf16(tmem + (uint32_t)x * 256u, t5::make_desc(al + o), t5::make_desc(bl + o), kPreIdescS, i > 0 ? 1u : 0u);
                    }
                    t5::commit(&sh.s_full[x]);
                };
                int look_view = 0, look_tail = 0;                         // a share's tiles with values to look at: one, and all from one on
                bool clean = false;                                       // the next tile to be multiplied has values to look at first
                uint32_t c_ph = 0;
                auto ask = [&](int j) {
                    clean = j == look_view || j >= look_tail;
                    if (ok && clean) ptx::mbar_arrive(&sh.v_ask);
                };
                auto half_product = [&](int x, int half, bool first) {
                    if (!ok) return;
                    t5::fence_after();
                    const uint32_t bl = (ring_lo + (uint32_t)vp.st * (kPreSlot >> 4)) | (kPreVStep << 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = half * 4 + i;
                        t5::mma_bf16_ta(tmem + (uint32_t)x * 256u + 128u, tmem + (uint32_t)x * 256u + (uint32_t)(k * 8),
                                        t5::make_desc(bl + (uint32_t)k * (2048u >> 4)), kPreIdescO, !first || k > 0 ? 1u : 0u);
                    }
                };
                int units = 0;                                            // of the share at hand; two: both row tiles have tokens
                bool two = false;
                auto open = [&]() {                                       // the next share that has tiles
                    while (walk.next(w, LG)) {
                        units = walk.units();
                        two = walk.rows2;
                        if (units == 0) continue;
                        look_view = walk.n_view % kPreTile ? walk.view_tiles - walk.t0 - 1 : -1;
                        look_tail = walk.view_tiles - walk.t0 + (walk.n_tail + walk.m0 + 1) / kPreTile;
                        return true;
                    }
                    return false;
                };
                bool have = open();
                if (have) {
                    if (ok) ok = ptx::mbar_wait(&sh.q_full, 0u) && ptx::mbar_wait(&sh.full[kp.st], kp.ph);
                    logits(0);
                    ask(0);
                    if (two) logits(1);
                    if (ok) t5::commit(&sh.empty[kp.st]);
                    if (ok && units == 1) t5::commit(&sh.q_empty);
                    kp.next();
                }
                while (have) {
                    const int n = units;
                    const bool both = two;
                    for (int j = 0; j < n; ++j) {
                        const bool more = j + 1 < n;
                        bool ahead = more;                                // a next tile: this share's, or the first of the next one
                        if (ok) ok = ptx::mbar_wait(&sh.full[vp.st], vp.ph);
                        // sums of the slots' last shares are out before new ones take their place (slot 1's too where it now rests: the flags of
                        // cleared values are kept for four shares)
                        if (j == 0) {
                            if (ok && out0 > 0) ok = ptx::mbar_wait(&sh.o_empty[0], (uint32_t)((out0 - 1) & 1));
                            if (ok && !both && out1 > 0) ok = ptx::mbar_wait(&sh.o_empty[1], (uint32_t)((out1 - 1) & 1));
                        }
                        if (clean) {
                            if (ok) ok = ptx::mbar_wait(&sh.v_clean, c_ph);
                            c_ph ^= 1u;
                        }
                        if (more) ask(j + 1);
                        if (ok) ok = ptx::mbar_wait(&sh.p_full[0][0], p_ph0);
                        half_product(0, 0, j == 0);
                        if (ok) t5::commit(&sh.h_full[0]);
                        if (ok) ok = ptx::mbar_wait(&sh.p_full[0][1], p_ph0);
                        half_product(0, 1, false);
                        p_ph0 ^= 1u;
                        if (!more) {
                            if (ok) t5::commit(&sh.o_full[0]);
                            ++seg;
                            ahead = have = open();
                            if (ok && ahead) ok = ptx::mbar_wait(&sh.q_full, (uint32_t)(seg & 1));
                        }
                        if (ahead) {
                            if (ok) ok = ptx::mbar_wait(&sh.full[kp.st], kp.ph);
                            logits(0);
                            if (!more) ask(0);
                        }
                        if (both) {
                            if (j == 0 && ok && out1 > 0) ok = ptx::mbar_wait(&sh.o_empty[1], (uint32_t)((out1 - 1) & 1));
                            if (ok) ok = ptx::mbar_wait(&sh.p_full[1][0], p_ph1);
                            half_product(1, 0, j == 0);
                            if (ok) t5::commit(&sh.h_full[1]);
                            if (ok) ok = ptx::mbar_wait(&sh.p_full[1][1], p_ph1);
                            half_product(1, 1, false);
                            p_ph1 ^= 1u;
                            if (ok && !more) t5::commit(&sh.o_full[1]);
                        }
                        if (ahead && two) logits(1);
                        if (ok) t5::commit(&sh.empty[vp.st]);
                        vp.next();
                        if (ahead) {
                            if (ok) t5::commit(&sh.empty[kp.st]);
                            if (ok && (more ? j + 2 == n : units == 1)) t5::commit(&sh.q_empty);
                            kp.next();
                        }
                    }
                    ++out0;
                    if (both) ++out1;
                }
                t5::commit(&sh.drained);                                  // MMAs in flight end before the tensor memory is given back
                ok = ptx::mbar_wait(&sh.drained, 0u) && ok;
                if (!ok) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
            }
        } else {
            // ------------------------------------------------ values that rows do not see: two warps
            const int ht = tid & 63;
            int tiles = 0, asked = 0, seg = 0;
            while (walk.next(w, LG)) {
                const int units = walk.units();
                if (units == 0) continue;
                for (int j = 0; j < units && ok; ++j) {
                    const int t = walk.t0 + j;
                    if (!walk.cleans(t)) continue;
                    // The MMA thread asks when the tile that was in this ring slot before has landed for certain (a wait for a phase two
                    // ahead of the barrier's would be over at once).
                    const int v = 2 * (tiles + j) + 1, st = v % RING;
                    ok = pre_wait_long(sh, &sh.v_ask, (uint32_t)(asked & 1)) && ptx::mbar_wait(&sh.full[st], (uint32_t)((v / RING) & 1));
                    ok = __all_sync(0xffffffffu, ok);
                    ++asked;
                    if (!ok) break;
                    unsigned char* vt = ring + (size_t)st * kPreSlot;
                    const int n_valid = walk.valid_of(t), first = max(walk.plain_of(t), 0);
                    auto at = [&](int i) {                                // 16 bytes of the tile, the swizzle's way
                        const int rr = i >> 4, c = i & 15;
                        return reinterpret_cast<uint4*>(vt + (size_t)(c >> 3) * kPreHalf + rr * 128 + (((c & 7) ^ (rr & 7)) << 4));
                    };
                    const int held = min(n_valid, kPreTile) * 16;
                    bool cleared = false;
#pragma unroll 4
                    for (int i = first * 16 + ht; i < held; i += 64) {
                        uint4 val = *at(i);
                        uint32_t* e = reinterpret_cast<uint32_t*>(&val);
                        __nv_bfloat162 any = __float2bfloat162_rn(0.0f);  // 0 x value summed up: NaN where one is not finite
#pragma unroll
                        for (int h = 0; h < 4; ++h) any = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&e[h]), __float2bfloat162_rn(0.0f), any);
                        if (__hbeq2(any, any)) continue;
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            if ((e[h] & 0x00007f80u) == 0x00007f80u) e[h] &= 0xffff0000u;
                            if ((e[h] & 0x7f800000u) == 0x7f800000u) e[h] &= 0x0000ffffu;
                        }
                        *at(i) = val;
                        cleared = true;
                    }
                    for (int i = max(held, 0) + ht; i < kPreTile * 16; i += 64) *at(i) = make_uint4(0u, 0u, 0u, 0u);
                    if (cleared) sh.not_finite[seg & 3] = seg + 1;
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.v_clean);
                }
                tiles += units;
                ++seg;
            }
            if (!ok && lane == 0) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 " PRE_ROW_REGS ";");
        // ------------------------------------------------ rows: a thread each
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t s_addr = tmem + (uint32_t)x * 256u + ((uint32_t)((warp & 3) * 32) << 16), o_addr = s_addr + 128u;
        const float scale2 = a.scale * 1.4426950408889634f;
        const int my_token = row / a.r, my_head = row - my_token * a.r;
        const int n_cta = sh.n_cta;
        int cnt = 0, done = 0, seg = 0;                  // units and shares of this slot; shares of the CTA
        auto wait = [&](uint64_t* bar, int phase) {
            if (ok) ok = ptx::mbar_wait(bar, (uint32_t)(phase & 1));
            ok = __all_sync(0xffffffffu, ok);
        };
        // The walk's state lies in shared memory, a copy a warp: beside a row's 128 logits there is no room for it in registers.
        PreWalk& walk = sh.walk[warp];
        if (lane == 0) walk = walk0;
        auto next = [&]() {
            __syncwarp();
            if (lane == 0) {
                PreWalk t = walk;
                t.more = t.next(w, LG);
                walk = t;
            }
            __syncwarp();
            return walk.more;
        };
        while (next()) {
            const int units = walk.units();
            const bool mine = x == 0 || walk.rows2;
            const int first_token = walk.m0 + x * tpt, token = first_token + my_token;
            const bool live = mine && my_token < tpt && token < walk.n_q;
            const int l = walk.clg / a.G, g = walk.clg % a.G;
            const size_t orow = (((size_t)walk.cs * a.M + token) * a.L + l) * a.H + (size_t)g * a.r + my_head;
            if (units == 0) {
                if (live) pre_zero_row(a, orow);
                continue;
            }
            if (mine) {
                const bool warp_live = __any_sync(0xffffffffu, live);
                float ref = -INFINITY, sum = 0.0f;
                // tokens that this row sees from the share's first tile on, as far as tiles are the view's, and behind
                const int view_units = walk.view_tiles - walk.t0, view_seen = walk.n_view - walk.t0 * kPreTile;
                const int tail_seen = walk.n_tail + min(token + 1, walk.n_q) + view_units * kPreTile;
                if (x == 1) {                                          // (slot 0 may have had shares to itself in between)
                    if (ok) ok = pre_wait_long(sh, &sh.s_full[1], (uint32_t)(cnt & 1));
                    ok = __all_sync(0xffffffffu, ok);
                }
                for (int j = 0; j < units; ++j) {
                    wait(&sh.s_full[x], cnt);
                    ++cnt;
                    if (warp_live) {
                        t5::fence_after();
                        uint32_t sv[4][32];
#pragma unroll
                        for (int c = 0; c < 4; ++c) t5::ld32_issue(s_addr + 32u * c, sv[c]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) t5::ld_wait(sv[c]);
                        // columns that this row sees: [0, seen)
                        const int seen = (j < view_units ? view_seen : tail_seen) - j * kPreTile;
                        if (__any_sync(0xffffffffu, seen < kPreTile)) {
#pragma unroll
                            for (int c = 0; c < 4; ++c)
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (32 * c + i >= seen) sv[c][i] = 0xff800000u;
                        }
                        const uint64_t sc2 = f2::pk(scale2, scale2);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            float part;
                            const float room = kPreLimit - sum;        // (known before the weights: sum + part behind them is 1,956 us, this 1,949)
                            for (bool again = false;; again = true) {
                                const float use = ref == -INFINITY ? 0.0f : ref;      // nothing seen yet: every weight is exp2(-inf) = 0
                                const uint64_t nm2 = f2::pk(-use, -use);
                                uint64_t acc0 = f2::pk(0.0f, 0.0f), acc1 = acc0;
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    uint32_t pk[16];
                                    const uint32_t (&v)[32] = sv[2 * half + c];
#pragma unroll
                                    for (int i = 0; i < 16; ++i) {
                                        float p0, p1;
                                        f2::unpk(f2::fma(f2::pk(v[2 * i], v[2 * i + 1]), sc2, nm2), p0, p1);
                                        p0 = t5::ex2(p0);
                                        p1 = t5::ex2(p1);
                                        if (i & 1) acc1 = f2::add(acc1, f2::pk(p0, p1)); else acc0 = f2::add(acc0, f2::pk(p0, p1));
                                        pk[i] = ptx::pack_bf16x2(p0, p1);         // what the tensor pipe takes beside bf16 values; the sum is of the fp32 weights
                                    }
                                    t5::st16(s_addr + 32u * half + 16u * c, pk);      // over logits that this thread has read
                                }
                                float a0, a1, a2, a3;
                                f2::unpk(acc0, a0, a1);
                                f2::unpk(acc1, a2, a3);
                                part = (a0 + a1) + (a2 + a3);
                                // rows without a reference yet, and those whose weights have grown past the limit (a NaN too)
                                const bool moves = live && (ref == -INFINITY || !(part <= room));
                                if (again || !__any_sync(0xffffffffu, moves)) break;
                                float m = -INFINITY;                   // largest logit of this half, NaN if one is
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    m = f2::max3_nan(m, __uint_as_float(sv[2 * half + (i >> 4)][2 * (i & 15)]), __uint_as_float(sv[2 * half + (i >> 4)][2 * (i & 15) + 1]));
                                m *= scale2;
                                const float so_far = ref + __log2f(sum);         // log2 of the row's sum in front of this half; -inf without one
                                m = f2::max3_nan(m, so_far, so_far);
                                const float to = moves && m != -INFINITY ? m : ref, corr = to == ref ? 1.0f : t5::ex2(ref - to);
                                // what O holds: the products before this tile's logits were issued, and the first half's
                                if (half == 1) {
                                    wait(&sh.h_full[x], cnt - 1);
                                    t5::fence_after();
                                }
                                if (j > 0 || half == 1) {
#pragma unroll 1
                                    for (int c = 0; c < 8; ++c) {
                                        uint32_t ov[16];
                                        t5::ld16_issue(o_addr + 16u * c, ov);
                                        t5::ld_wait(ov);
#pragma unroll
                                        for (int i = 0; i < 16; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * corr);
                                        t5::st16(o_addr + 16u * c, ov);
                                    }
                                }
                                sum *= corr;
                                ref = to;
                            }
                            sum += part;
                            t5::st_wait();
                            t5::fence_before();
                            if (half == 0) {                       // the first half of the tokens is ready for its product
                                __syncwarp();
                                if (lane == 0) ptx::mbar_arrive(&sh.p_full[x][0]);
                            }
                        }
                    } else if (lane == 0) {
                        ptx::mbar_arrive(&sh.p_full[x][0]);
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.p_full[x][1]);
                }
                // the share's sums
                wait(&sh.o_full[x], done++);
                const bool whole = walk.t0 == 0 && walk.t1 == walk.tiles;
                const int share = 2 * ((walk.part - 1) * n_cta + (int)blockIdx.x) + (walk.t0 == 0 ? 1 : 0);
                const bool nf = *(volatile int*)&sh.not_finite[seg & 3] == seg + 1;
                if (warp_live) {
                    t5::fence_after();
                    const bool none = sum == 0.0f;
                    if (whole) {
                        // 64 dims of each row at a time through the warp's staging, so that eight lanes write a row's 128 bytes together (a
                        // lane with 16 bytes of a row of its own takes eight times as many cycles of the store path)
                        const uint32_t stage = ptx::smem_u32(staging + warp * kPreStage);
                        const float inv = none ? 0.0f : 1.0f / sum;
                        unsigned long long to[8];                      // the rows that this lane writes a part of; 0: none
                        {
                            const unsigned long long mine_to = live ? (unsigned long long)(a.out + orow * kPreD) : 0ull;
#pragma unroll
                            for (int i = 0; i < 8; ++i) to[i] = __shfl_sync(0xffffffffu, mine_to, i * 4 + (lane >> 3));
                        }
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t ov[2][32], pk[32];
                            t5::ld32_issue(o_addr + 64u * c, ov[0]);
                            t5::ld32_issue(o_addr + 64u * c + 32u, ov[1]);
                            t5::ld_wait(ov[0]);
                            t5::ld_wait(ov[1]);
                            float* o = reinterpret_cast<float*>(ov);
#pragma unroll
                            for (int i = 0; i < 32; ++i) f2::unpk(f2::mul(f2::pk(o[2 * i], o[2 * i + 1]), f2::pk(inv, inv)), o[2 * i], o[2 * i + 1]);
                            if (nf && live && !none) {
                                // values that were cleared and that this row sees
                                for (int tok = walk.m0 + 1; tok <= token; ++tok) {
                                    const __nv_bfloat16* vr = a.tail_v + (((size_t)walk.cs * a.tail_cap + walk.n_tail + tok) * LG + walk.clg) * kPreD + 64 * c;
#pragma unroll
                                    for (int i = 0; i < 64; ++i) {
                                        const float v = __bfloat162float(vr[i]);
                                        if (!isfinite(v)) o[i] += v;
                                    }
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) pk[i] = none ? 0u : ptx::pack_bf16x2(o[2 * i], o[2 * i + 1]);
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + 128u * lane + 16u * (i ^ (lane & 7))), "r"(pk[4 * i]), "r"(pk[4 * i + 1]), "r"(pk[4 * i + 2]), "r"(pk[4 * i + 3]) : "memory");
                            __syncwarp();
                            uint32_t vv[8][4];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const int rr = i * 4 + (lane >> 3);
                                uint32_t (&v)[4] = vv[i];
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(stage + 128u * rr + 16u * ((lane & 7) ^ (rr & 7))) : "memory");
                            }
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (to[i]) asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(to[i] + 128 * c + 16 * (lane & 7)), "r"(vv[i][0]), "r"(vv[i][1]), "r"(vv[i][2]), "r"(vv[i][3]) : "memory");
                        }
                        if (live) a.lse[orow] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
                    } else {
                        // partial sums lie four dims at a time, a row's behind another's: a warp's stores are whole lines as they are
                        float4* po = reinterpret_cast<float4*>(w.part_o) + ((size_t)share * 2 + x) * (kPreD / 4) * kPreRows + row;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t ov[32];
                            t5::ld32_issue(o_addr + 32u * c, ov);
                            t5::ld_wait(ov);
                            if (live) {
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    po[(size_t)(8 * c + i) * kPreRows] = make_float4(__uint_as_float(ov[4 * i]), __uint_as_float(ov[4 * i + 1]), __uint_as_float(ov[4 * i + 2]), __uint_as_float(ov[4 * i + 3]));
                            }
                            __syncwarp();
                        }
                        if (live) w.part_ml[(size_t)share * 2 * kPreRows + x * kPreRows + row] = make_float2(ref, sum);
                    }
                    t5::fence_before();
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.o_empty[x]);
                if (!whole && tid == 0) {
                    const int all = n_cta * sh.n_parts;
                    w.rec[share] = PreRecord{walk.cs, walk.clg, walk.crg, (int)(((unsigned long long)(walk.last + 1) * all - 1) / sh.total)};
                    w.nf[share] = nf;
                }
            }
            ++seg;
        }
        if (!ok && lane == 0) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
    }
    t5::fence_before();
    __syncthreads();
    if (warp == kPreMmaWarp) {
        t5::fence_after();
        t5::tmem_dealloc(tmem, 512);
    }
}

// Joins the shares of the items that cuts of the line fall into, in line order: for every part c, the item whose first cut is the part's
// start, if there is one.  The grid's first axis goes over the parts, the second is the slot and 32 of the dims.  A warp has 32 rows, a
// lane each, and 16 dims: its reads are whole lines.  Bound by latency (a round of dependent reads costs some 0.6 us): two shares
// are requested together, and blocks go on to the next part rather than be many and mostly empty.
constexpr int kPreMergeThreads = 256, kPreMergeBatch = 2;
__global__ void __launch_bounds__(kPreMergeThreads, 4)
prefill_merge_kernel(const __grid_constant__ PreWork w) {
    pdl_wait();
    pdl_trigger();
    const PrefillArgs& a = w.a;
    const int warp = threadIdx.x >> 5, x = blockIdx.y >> 2, n_parts = *w.n_parts;
    for (int c = blockIdx.x + 1; c < n_parts; c += gridDim.x) {
        const PreRecord it = w.rec[2 * c], head = w.rec[2 * c - 1];
        if (it.s < 0 || head.s != it.s || head.lg != it.lg || head.rg != it.rg) continue;
        const int LG = a.L * a.G, m0 = it.rg * 2 * w.tpt, first_token = m0 + x * w.tpt, shares = it.last - c + 2;
        const int n_q = a.n_q ? min(max(a.n_q[it.s], 0), a.M) : a.M;
        const int rows = min(w.tpt, n_q - first_token) * a.r;               // live ones of this row tile
        const int row = (warp & 3) * 32 + (threadIdx.x & 31), d0 = (blockIdx.y & 3) * 32 + (warp >> 2) * 16;
        if (row >= rows) continue;
        auto share = [&](int i) { return i == 0 ? 2 * c - 1 : 2 * (c - 1 + i); };
        float top = -INFINITY, z = 0.0f;
        float4 acc[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        int nf = 0;
        for (int i0 = 0; i0 < shares; i0 += kPreMergeBatch) {
            float2 ml[kPreMergeBatch];
            float4 v[kPreMergeBatch][4];
#pragma unroll
            for (int i = 0; i < kPreMergeBatch; ++i) {
                ml[i] = make_float2(-INFINITY, 0.0f);
                if (i0 + i < shares) {
                    ml[i] = w.part_ml[(size_t)share(i0 + i) * 2 * kPreRows + x * kPreRows + row];
                    nf |= w.nf[share(i0 + i)];
                    const float4* po = reinterpret_cast<const float4*>(w.part_o) + (((size_t)share(i0 + i) * 2 + x) * (kPreD / 4) + d0 / 4) * kPreRows + row;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[i][k] = po[(size_t)k * kPreRows];
                }
            }
            float to = top;
#pragma unroll
            for (int i = 0; i < kPreMergeBatch; ++i) to = fmaxf(to, ml[i].x + __log2f(ml[i].y));      // (by its sum: no share is more than its values)
            const float back = top > -INFINITY ? t5::ex2(top - to) : 1.0f;            // (without a reference z and acc are 0, or NaN)
            z *= back;
#pragma unroll
            for (int k = 0; k < 4; ++k) { acc[k].x *= back; acc[k].y *= back; acc[k].z *= back; acc[k].w *= back; }
#pragma unroll
            for (int i = 0; i < kPreMergeBatch; ++i)
                if (ml[i].x > -INFINITY || ml[i].y != 0.0f) {                          // a share without a visible token holds no sums
                    const float f = t5::ex2(ml[i].x - to);
                    z += f * ml[i].y;
#pragma unroll
                    for (int k = 0; k < 4; ++k) { acc[k].x += f * v[i][k].x; acc[k].y += f * v[i][k].y; acc[k].z += f * v[i][k].z; acc[k].w += f * v[i][k].w; }
                }
            top = to;
        }
        const int token = first_token + row / a.r;
        const bool none = z == 0.0f;
        const float inv = none ? 0.0f : 1.0f / z;
        float out[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            out[4 * k] = none ? 0.0f : acc[k].x * inv; out[4 * k + 1] = none ? 0.0f : acc[k].y * inv;
            out[4 * k + 2] = none ? 0.0f : acc[k].z * inv; out[4 * k + 3] = none ? 0.0f : acc[k].w * inv;
        }
        if (nf && !none) {
            const int n_tail = min(max(a.n_tail[it.s], 0), a.tail_cap - n_q);
            for (int tok = m0 + 1; tok <= token; ++tok) {
                const __nv_bfloat16* vr = a.tail_v + (((size_t)it.s * a.tail_cap + n_tail + tok) * LG + it.lg) * kPreD + d0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = __bfloat162float(vr[i]);
                    if (!isfinite(v)) out[i] += v;
                }
            }
        }
        const size_t orow = (((size_t)it.s * a.M + token) * a.L + it.lg / a.G) * a.H + (size_t)(it.lg % a.G) * a.r + row % a.r;
        uint32_t pk[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) pk[i] = ptx::pack_bf16x2(out[2 * i], out[2 * i + 1]);
        uint4* dst = reinterpret_cast<uint4*>(a.out + orow * kPreD + d0);
        dst[0] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
        dst[1] = make_uint4(pk[4], pk[5], pk[6], pk[7]);
        if (d0 == 0) a.lse[orow] = none ? -INFINITY : (top + log2f(z)) * 0.6931471805599453f;
    }
}

static size_t plan_prefill(char* base, PreWork* w) {
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return base ? base + at : nullptr; };
    constexpr size_t shares = (size_t)kSMs * kPreParts * 2;
    w->part_o = (float*)take(shares * 2 * kPreRows * kPreD * sizeof(float));
    w->part_ml = (float2*)take(shares * 2 * kPreRows * sizeof(float2));
    w->rec = (PreRecord*)take(shares * sizeof(PreRecord));
    w->nf = (int*)take(shares * sizeof(int));
    w->n_parts = (int*)take(sizeof(int));
    return off;
}

size_t prefill_workspace_bytes(const kvmem_pool_config_t&) {
    PreWork w;
    return plan_prefill(nullptr, &w);
}

static long long pre_most_units(const kvmem_pool_config_t& c, int n_sessions, int n_q_tokens, int cap, int tail_cap) {
    const int tpt = kPreRows / (c.n_q_heads / c.n_kv_heads);
    const long long groups = (n_q_tokens + 2ll * tpt - 1) / (2 * tpt);
    const long long tiles = ((long long)cap + kPreTile - 1) / kPreTile + ((long long)tail_cap + kPreTile - 1) / kPreTile + 1 + kPreLead;
    return (long long)n_sessions * c.n_layers * c.n_kv_heads * groups * tiles;
}

// the line in 30 bits, row groups of a head in 16, token rows in the 32 bits of a TMA coordinate
bool prefill_fits(const kvmem_pool_config_t& c, int n_sessions, int n_q_tokens, int cap_tokens, int tail_cap_tokens) {
    const int tpt = kPreRows / (c.n_q_heads / c.n_kv_heads);
    return (long long)n_q_tokens <= 65535ll * 2 * tpt && (long long)n_sessions * n_q_tokens < INT32_MAX - 256 &&
           (long long)n_sessions * c.n_layers * c.n_kv_heads < (1 << 30) &&
           (double)pre_most_units(c, n_sessions, n_q_tokens, cap_tokens, tail_cap_tokens) < (double)kPreMostUnits;
}

static bool pre_map(CUtensorMap* map, const __nv_bfloat16* p, cuuint64_t d1, cuuint64_t d2, cuuint32_t box1, cuuint32_t box2) {
    static PFN_cuTensorMapEncodeTiled_v12000 enc = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr) : nullptr;
    }();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)kPreD, d1, d2};
    cuuint64_t strides[2] = {(cuuint64_t)kPreD * 2, d1 * kPreD * 2};
    cuuint32_t box[3] = {64, box1, box2}, step[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_prefill(const kvmem_pool& p, const PrefillArgs& a, void* workspace, cudaStream_t st) {
    static PerDeviceOnce once;
    if (once.pending(p.cfg.device)) {
        const cudaError_t e = cudaFuncSetAttribute(prefill_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPreSmem);
        if (e != cudaSuccess) return e;
        once.mark(p.cfg.device);
    }
    PreWork w{};
    plan_prefill((char*)workspace, &w);
    w.a = a;
    w.tpt = kPreRows / a.r;
    w.log_group = -1;
    for (int i = 0; i <= 8; ++i)
        if (2 * w.tpt == 1 << i) w.log_group = i;
    const int LG = a.L * a.G;
    CUtensorMap mq, mk, mv, mtk, mtv;
    bool made = pre_map(&mq, a.q, (cuuint64_t)a.L * a.H, (cuuint64_t)a.ns * a.M, (cuuint32_t)a.r, (cuuint32_t)w.tpt) &&
                pre_map(&mk, a.view_k, (cuuint64_t)a.cap, (cuuint64_t)a.ns * LG, kPreTile, 1) &&
                pre_map(&mv, a.view_v, (cuuint64_t)a.cap, (cuuint64_t)a.ns * LG, kPreTile, 1);
    if (a.tail_k)
        made = made && pre_map(&mtk, a.tail_k, (cuuint64_t)LG, (cuuint64_t)a.ns * a.tail_cap, 1, kPreTile) &&
               pre_map(&mtv, a.tail_v, (cuuint64_t)LG, (cuuint64_t)a.ns * a.tail_cap, 1, kPreTile);
    else { mtk = mk; mtv = mv; }
    if (!made) return cudaErrorInvalidValue;
    const int grid = (int)std::min<long long>(std::min(p.sm_count, kSMs), pre_most_units(p.cfg, a.ns, a.M, a.cap, a.tail_cap));
    cudaError_t e = launch_pdl(prefill_kernel, dim3((unsigned)grid), dim3(kPreThreads), kPreSmem, st, mq, mk, mv, mtk, mtv, w);
    // as many parts as the line can have
    const long long units = pre_most_units(p.cfg, a.ns, a.M, a.cap, a.tail_cap);
    const long long parts = std::min(units, grid * std::max(1ll, std::min<long long>(kPreParts, units / ((long long)grid * kPrePartUnits))));
    if (e != cudaSuccess || parts < 2) return e;
    return launch_pdl(prefill_merge_kernel, dim3((unsigned)std::min<long long>(parts - 1, grid), 8), dim3(kPreMergeThreads), 0, st, w);
}

}  // namespace kvmem
