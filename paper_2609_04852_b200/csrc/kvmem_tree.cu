// Attention of drafted tokens over a view (or the selected pages) and the tail of tokens behind it, and the weights it
// leaves on the view:   out_i = sum_t p_it v_t,  p_it = exp(x_it - lse_i),  x_it = scale q_i . k_t over the t that i sees,
//                       mass_t = decay mass_t + sum_i p_it.
//
// The query rows of a KV head (drafted tokens x query heads that share it) are the rows of one or two 128-row tiles, the
// tokens come in tiles of 128: view tiles first, then tail tiles (committed and drafted tokens).  Per tile
//     S = Q K^T   tcgen05.mma, both operands in shared memory, 128 x 128 fp32 accumulators in tensor memory
//     P = exp2(S scale log2e - ref)   two threads per row (TMEM lane), each with half of the columns: no shuffles
//     O += P V    tcgen05.mma, P as bf16 in tensor memory (in the place of S), V from shared memory
// Two slots (S, P and O each: 2 x 256 columns, all of tensor memory) keep the tensor pipe and the special-function unit
// busy in turn: with up to 128 rows the slots take tiles alternately and are merged at the end like two splits; with more
// rows slot w is row tile w and both read the same K and V tile.  Two warps fetch tiles with TMA (128-byte swizzle), one the
// keys and one the values, into a ring of 32 KiB slots, one thread issues the MMAs, sixteen warps hold the rows.
//
// ref is a running maximum that moves only when a row's logits pass it by 8 (in powers of two): O is then rescaled in
// tensor memory.  Until then the weights may reach 2^8, which costs neither fp32 nor bf16 any precision.
//
// Work: the tiles of all (session, KV head, row group) lie on one line, with a lead of a few tiles' time ahead of each head for
// the switch, cut into as many equal parts as there are CTAs (one per SM), so that sessions of any lengths keep all SMs busy
// to the end.  A CTA's share of one head is a segment;
// each leaves unnormalised sums, row references and row sums, and tree_merge_kernel joins a head's segments in order: the
// result depends on the sizes alone, not on timing.  Lengths are read on the device.
//
// Tokens that nobody may see: their logits are replaced before they are used, and their values are cleared in shared
// memory before the second product (0 x NaN).  A drafted token's value that is not finite would reach the tokens that do
// not see it in the same way: such elements are cleared too, and the merge adds them to the rows that see them.
#include <cudaTypedefs.h>
#include <math.h>

#include <algorithm>

#include "kvmem_internal.cuh"
#include "kvmem_ptx.cuh"
#include "kvmem_t5.cuh"

namespace kvmem {

constexpr int kTreeD = 128;
constexpr int kTreeTile = 128;                    // tokens per tile
constexpr int kTreeHalf = kTreeTile * 128;        // bytes of one 64-dim half of a 128-row operand tile (16 KiB)
constexpr int kTreeSlot = 2 * kTreeHalf;          // a K, V or Q tile
constexpr int kTreeRows = 128;                    // rows of a row tile: TMEM lanes
constexpr int kTreeThreads = 32 * 19;              // key and value TMA warps, MMA warp, sixteen row warps
constexpr int kTreeVWarp = 18;
// Ring slots, K and V tiles in turn: two tiles of each per SM, 18.5 MiB over the 148.  There is room for six slots beside one Q
// tile, but more requests than HBM's latency asks for only lengthen its queues: eight sessions of up to 65,536 tokens take 177 us
// with four slots and 184 with six, 262,144 tokens with the weights of 16 rows 225 and 240, 32,768 tokens 34.6 and 35.2 (SM clock at
// 1,965 MHz; under the power limit 192 and 191, 234 and 245, 34.9 and 35.4).
constexpr int kTreeRing = 4;
constexpr float kTreeSlack = 8.0f;                // a row's logits may pass its reference by this much (log2)
constexpr uint32_t kTreeIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (16u << 17) | (8u << 24);   // bf16 x bf16 -> fp32, 128 x 128
constexpr uint32_t kTreeIdescO = kTreeIdescS | (1u << 16);                                        // B with dims contiguous (V as it lies)
constexpr uint32_t kTreeVStep = (uint32_t)kTreeHalf >> 4;      // leading offset of V's descriptor: from dims 0..63 to 64..127

struct TreeSpan {
    int n_view, n_tail, n_q;      // view tokens, committed tail tokens, drafted tokens of the session
    int view_tiles, tiles;        // tiles of the view, tiles of view and tail
    int groups;                   // row groups per KV head: up to two row tiles each
};

// What the merge needs to know of a session: where it starts on the line, its tiles, row groups, drafted and committed tokens.
// Entry ns: the line's length, the CTAs that share it, a head's lead.
struct TreeInfo {
    int start, tiles, groups, n_q, n_tail;
};

struct TreeWork {
    TreeArgs a;
    int row_groups, rows_slot;    // most row groups a head can have, rows stored per slot
    float* part_o;                // [segment][slot][rows_slot][128]
    float2* part_ml;              // [segment][slot][rows_slot]: (reference, sum of weights), log2 domain
    ulonglong2* part_nf;          // [segment]: a byte per row warp, set where it cleared a drafted value that is not finite
    TreeInfo* info;               // [ns + 1], filled by CTA 0
    float* lse2;                  // [ns][LG][rows]: log-sum-exp in the log2 domain, +inf where it is -inf (weights only)
    float* logits;                // [ns][LG][rows][cap]: scaled logits, log2 domain (weights only)
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
    t.view_tiles = (t.n_view + kTreeTile - 1) / kTreeTile;
    t.groups = (t.n_q * a.r + 2 * kTreeRows - 1) / (2 * kTreeRows);
    t.tiles = t.n_q > 0 ? t.view_tiles + (a.tail_k ? (t.n_tail + t.n_q + kTreeTile - 1) / kTreeTile : 0) : 0;
    return t;
}

// drafted tokens that drafted token m sees, those in use only
__device__ __forceinline__ unsigned long long tree_bits(const TreeArgs& a, int s, int m, int n_q) {
    const unsigned long long all = n_q >= 64 ? ~0ull : (1ull << n_q) - 1;
    return all & (a.mask ? a.mask[(size_t)s * a.M + m] : (m >= 63 ? ~0ull : (2ull << m) - 1));
}

// columns [c0, c0 + 32) of a tail tile that a row sees: committed tokens, then its drafted ones
__device__ __forceinline__ uint32_t tail_word(int c0, int n_tail, unsigned long long bits) {
    const int d = n_tail - c0;                       // column of drafted token 0
    const uint32_t committed = d >= 32 ? 0xffffffffu : d <= 0 ? 0u : (1u << d) - 1u;
    const uint32_t drafted = d >= 32 || d <= -64 ? 0u : d >= 0 ? (uint32_t)(bits << d) : (uint32_t)(bits >> -d);
    return committed | drafted;
}

// row tiles of row group rg when the session has `rows` live rows: with one, the slots take tiles in turn
__device__ __forceinline__ int tree_row_tiles(int rows, int rg) { return rows - rg * 2 * kTreeRows > kTreeRows ? 2 : 1; }

// The line: per (session, KV head, row group) `lead` units that stand for what going on to another head costs a CTA, and units for
// its tiles; CTA c of n has the tiles that begin in units [total c / n, total (c + 1) / n).  A tile is one unit; in a call
// where heads may have two row tiles (wide: more than 128 rows) one with two is two, and a part is two units or more, so that no
// CTA between two others of a head is left without a tile of it.  (All tiles alike: 53 us instead of 49 for rows of 256 + 8, 64
// instead of 55 for 256 + 128, 24,864 tokens, 8 heads; the longer walk costs calls of 192 or 256 rows 1.5 to 5 %.)  The leads, in
// us: eight ragged sessions of up to 24,896 tokens, 8 heads, take 75.5, 72.1, 71.9, 72.4 with a lead of 1, 2, 3, 5 at 4 rows and 82.3,
// 80.1, 77.9, 76.5 at 48; two sessions of 24,896 and 19,264, 2 layers, 4 heads (wide) 60.9, 58.8, 57.9, 57.4 with 3, 5, 8, 12 at 136
// rows, 67.3, 65.3, 63.8, 63.3 at 192, 69.7, 68.0, 66.7, 64.9 at 256, and the same within the noise of some 5 % at 264 to 512.
// The host refuses calls that could pass 2^30 units (tree_line_fits).
constexpr int kTreeMostUnits = 1 << 30;
constexpr __host__ __device__ int tree_lead(bool wide) { return wide ? 8 : 3; }
constexpr __host__ __device__ int tree_most(bool wide) { return wide ? 2 : 1; }     // units of a tile at most
// of a session, in a wide call
struct TreeCosts {
    int shift;         // log2 of the units of a tile of the last row group; the ones before it have two row tiles
    int full, head;    // units of a row group before the last, of the KV head
    __device__ __forceinline__ TreeCosts(const TreeSpan& sp, int r, int lead) {
        shift = tree_row_tiles(sp.n_q * r, sp.groups - 1) - 1;
        full = 2 * sp.tiles + lead;
        head = (sp.groups - 1) * full + (sp.tiles << shift) + lead;
    }
};

// x * m / d; the product fits 32 bits in any call that fits the memory, and a division of 64 bits takes several times as long
__device__ __forceinline__ int mul_div(int x, int m, int d) {
    const unsigned long long p = (unsigned long long)x * (unsigned)m;
    return p < (1ull << 32) ? (int)((unsigned)p / (unsigned)d) : (int)(p / (unsigned)d);
}
__device__ __forceinline__ int line_owner(int x, int total, int n) {
    const unsigned long long p = (unsigned long long)(x + 1) * (unsigned)n - 1u;
    return p < (1ull << 32) ? (int)((unsigned)p / (unsigned)total) : (int)(p / (unsigned)total);
}

// a role's walk over the CTA's segments
struct TreeWalk {
    int pos, end, base, lead;     // next unit of the line, the CTA's end, first unit of session s
    int s, lg, rg, head, t0, t1;  // the segment: tiles [t0, t1) of head `head` (a row group of a KV head)
    int qt;                       // its row tiles
    TreeSpan sp;
    template <bool WIDE>
    __device__ __forceinline__ bool next(const TreeArgs& a, int most_groups) {
        const int LG = a.L * a.G;
        while (pos < end) {
            sp = tree_span(a, s, false);
            while (true) {
                const int units = sp.tiles ? (WIDE ? TreeCosts(sp, a.r, lead).head : sp.tiles + lead) * LG : 0;
                if (base + units > pos) break;
                base += units;
                sp = tree_span(a, ++s, false);
            }
            int from, shift = 0;                              // unit of the row group's first tile; a tile is 2^shift units
            rg = 0;
            if (WIDE) {
                const TreeCosts u(sp, a.r, lead);
                lg = (pos - base) / u.head;
                from = base + lg * u.head;
                if (sp.groups > 1) rg = min((pos - from) / u.full, sp.groups - 1);
                shift = rg == sp.groups - 1 ? u.shift : 1;
                from += rg * u.full + lead;
            } else {
                lg = (pos - base) / (sp.tiles + lead);
                from = base + lg * (sp.tiles + lead) + lead;
            }
            const int up = (1 << shift) - 1;
            t0 = (max(pos - from, 0) + up) >> shift;
            t1 = min(sp.tiles, WIDE ? (max(end - from, 0) + up) >> shift : end - from);
            pos = min(end, from + (sp.tiles << shift));
            if (t0 >= t1) continue;                           // nothing but the head's lead
            head = (s * LG + lg) * most_groups + rg;
            qt = shift + 1;
            return true;
        }
        return false;
    }
};

// 32 logits of a row to weights exp2(x scale2 - ref), bf16 pairs in pk; their fp32 sum goes to acc0 + acc1.  (A quarter of the
// exponentials as a polynomial on the FMA pipe, as chunked scoring has it, gains nothing: the unit waits for the MMAs.)
__device__ __forceinline__ void tree_weights(const uint32_t (&sv)[32], uint64_t sc2, uint64_t nm2, uint64_t& acc0, uint64_t& acc1, uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float p0, p1;
        f2::unpk(f2::fma(f2::pk(sv[2 * i], sv[2 * i + 1]), sc2, nm2), p0, p1);
        p0 = t5::ex2(p0);
        p1 = t5::ex2(p1);
        if (i & 1) acc1 = f2::add(acc1, f2::pk(p0, p1)); else acc0 = f2::add(acc0, f2::pk(p0, p1));
        pk[i] = ptx::pack_bf16x2(p0, p1);
    }
}

struct TreeShared {
    uint64_t full[kTreeRing], empty[kTreeRing], q_full, s_full[2], p_full[2], o_done[2], drained;
    int plan_begin, plan_end, plan_base, plan_s, plan_lead;
    uint32_t tmem;
    float half_max[2][2][kTreeRows];      // [slot][half of the columns]: exchanged between the two threads of a row
};
// Nothing static beside it: the dynamic part then starts where shared memory does, on the 1,024 bytes that the swizzle needs
// (checked).
constexpr size_t tree_smem(int q_tiles) { return (size_t)(q_tiles + kTreeRing) * kTreeSlot + sizeof(TreeShared); }

template <int QT, bool PAGED, bool MASS>
__global__ void __launch_bounds__(kTreeThreads, 1)
tree_split_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_tk, const __grid_constant__ CUtensorMap map_tv,
                  const __grid_constant__ TreeWork w) {
    constexpr int RING = kTreeRing;
    extern __shared__ __align__(1024) unsigned char smem_q[];      // Q tiles, the ring, then the small things
    const TreeArgs& a = w.a;
    unsigned char* ring = smem_q + (size_t)QT * kTreeSlot;
    TreeShared& sh = *reinterpret_cast<TreeShared*>(ring + (size_t)RING * kTreeSlot);
    uint64_t *full = sh.full, *empty = sh.empty, *s_full = sh.s_full, *p_full = sh.p_full, *o_done = sh.o_done;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int LG = a.L * a.G;

    if (ptx::smem_u32(smem_q) & 1023u) {          // never: see TreeShared
        if (tid == 0) atomicExch(a.status, (int)KVMEM_E_UNSUPPORTED);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < RING; ++i) { ptx::mbar_init(&full[i], 1); ptx::mbar_init(&empty[i], 1); }
        for (int i = 0; i < 2; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&p_full[i], 8); ptx::mbar_init(&o_done[i], 1); }
        ptx::mbar_init(&sh.q_full, 16);
        ptx::mbar_init(&sh.drained, 1);
        ptx::fence_mbar_init();
    }
    if (tid == 32 * kTreeVWarp) {
        ptx::prefetch_tensormap(&map_k);
        if (!PAGED) ptx::prefetch_tensormap(&map_v);
        if (a.tail_k) { ptx::prefetch_tensormap(&map_tk); ptx::prefetch_tensormap(&map_tv); }
    }
    if (warp == 1) {
        t5::tmem_alloc(&sh.tmem, 512);
        t5::tmem_relinquish();
    }
    pdl_wait();        // everything earlier in the stream is complete and visible from here on
    pdl_trigger();
    if (warp == 0) {
        // the CTA's part of the line, and the session it starts in
        constexpr bool WIDE = QT == 2;
        int sum = 0, live = 0, lo_t = INT32_MAX, hi_t = 0;    // one KV head of all sessions: units of tiles, row groups; units of a row group
#pragma unroll 4
        for (int s = lane; s < a.ns; s += 32) {
            const TreeSpan sp = tree_span(a, s, blockIdx.x == 0);
            const int heads = sp.tiles ? sp.groups : 0;
            if (WIDE) {
                const TreeCosts u(sp, a.r, 0);
                sum += heads ? u.head : 0;
                lo_t = min(lo_t, sp.tiles << u.shift);
                hi_t = max(hi_t, heads > 1 ? u.full : sp.tiles << u.shift);
            } else {
                sum += sp.tiles * heads;
                lo_t = min(lo_t, sp.tiles);
                hi_t = max(hi_t, sp.tiles);
            }
            live += heads;
        }
        if (a.ns > 1) {
            sum = __reduce_add_sync(0xffffffffu, sum);
            live = __reduce_add_sync(0xffffffffu, live);
            lo_t = __reduce_min_sync(0xffffffffu, lo_t);
            hi_t = __reduce_max_sync(0xffffffffu, hi_t);
        } else {
            sum = __shfl_sync(0xffffffffu, sum, 0); live = __shfl_sync(0xffffffffu, live, 0);
            lo_t = __shfl_sync(0xffffffffu, lo_t, 0); hi_t = __shfl_sync(0xffffffffu, hi_t, 0);
        }
        const int heads = live * LG, tiles = sum * LG;
        int lead = heads > 1 ? tree_lead(WIDE) : 0, n = min((int)gridDim.x, (tiles + tree_most(WIDE) - 1) / tree_most(WIDE));
        // Heads of one length: with a multiple of their number of CTAs none has parts of two heads.  That costs a few SMs and saves
        // the switches; the better of the two.
        if (lo_t == hi_t && heads > 0 && heads <= gridDim.x) {
            const int per_head = min((int)gridDim.x / heads, max(hi_t / tree_most(WIDE), 1));
            if ((hi_t + per_head - 1) / per_head <= (tiles + n - 1) / n + tree_lead(WIDE)) { n = per_head * heads; lead = 0; }
        }
        const int total = tiles + heads * lead;
        const bool idle = (int)blockIdx.x >= n;
        const int begin = idle ? 0 : mul_div(total, blockIdx.x, n), end = idle ? 0 : mul_div(total, blockIdx.x + 1, n);
        int before = 0;
        for (int s0 = 0; s0 < a.ns; s0 += 32) {
            const int s = s0 + lane;
            TreeSpan sp{};
            if (s < a.ns) sp = tree_span(a, s, false);
            const int mine = sp.tiles ? (WIDE ? TreeCosts(sp, a.r, lead).head : sp.tiles + lead) * LG : 0;
            int incl = mine;
            if (a.ns > 1) {
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += up;
                }
            }
            const int lo = before + incl - mine;
            if (begin >= lo && begin < lo + mine) { sh.plan_s = s; sh.plan_base = lo; }
            if (blockIdx.x == 0 && s < a.ns) w.info[s] = TreeInfo{lo, sp.tiles, sp.groups, sp.n_q, sp.n_tail};
            before += __shfl_sync(0xffffffffu, incl, 31);
            if (blockIdx.x != 0 && (idle || before > begin)) break;
        }
        if (lane == 0) {
            sh.plan_begin = begin;
            sh.plan_end = end;
            sh.plan_lead = lead;
            if (blockIdx.x == 0) w.info[a.ns] = TreeInfo{total, n, lead, 0, 0};
        }
    }
    // warp 0 has what it needs and goes on; the others wait for the plan and the tensor memory
    t5::fence_before();
    if (warp == 0) {
        __syncwarp();
        asm volatile("bar.arrive 10, %0;" ::"n"(kTreeThreads) : "memory");
    } else {
        asm volatile("bar.sync 10, %0;" ::"n"(kTreeThreads) : "memory");
    }
    t5::fence_after();
    const uint32_t tmem = warp == 0 ? 0u : sh.tmem;
    TreeWalk walk;
    walk.pos = sh.plan_begin; walk.end = sh.plan_end; walk.base = sh.plan_base; walk.s = sh.plan_s; walk.lead = sh.plan_lead;

    // A wait that runs out is recorded and the role goes on without waiting (and without issuing what would need it), so that
    // every role still reaches its end.
    bool ok = true;
    if (warp == 0 || warp == kTreeVWarp) {
        // ------------------------------------------------ TMA: warp 0 the keys, the last warp the values, each with every second
        // load of the ring
        const int kv = warp == 0 ? 0 : 1;
        const CUtensorMap *map_in = PAGED || kv == 0 ? &map_k : &map_v, *map_tail = kv ? &map_tv : &map_tk;
        const uint64_t once = ptx::l2_evict_first();          // keys and values make room for the partial sums: 41 -> 38 us at 32,768 tokens
        int n = kv;                                           // next load
        const int box = PAGED ? min(a.B, 64) : 64;            // tokens per copy
        const int boxes = kTreeTile / box, per_block = PAGED ? max(a.B / 64, 1) : 1;     // copies per tile, per block
        while (walk.next<(QT == 2)>(a, w.row_groups)) {
            const int n_box = (walk.sp.n_view + box - 1) / box;           // copies that hold view tokens
            const int b_end = min(n_box, min(walk.t1, walk.sp.view_tiles) * boxes);
            const int NB = PAGED ? a.nblocks_dev[a.session_first + walk.s] : 0;
            // page of the block that copy b reads: two dependent loads, 32 copies at a time and a batch ahead
            auto lookup = [&](int b) -> int {
                if (!PAGED || b >= b_end) return -1;
                const int id = a.sel_ids[(size_t)walk.s * a.sel_stride + (per_block == 1 ? b : b / per_block)];
                int pg = -1;
                if (id >= 0 && id < NB) pg = a.tables[(size_t)(a.session_first + walk.s) * a.max_bps + id];
                if (pg < 0 || pg >= a.max_blocks) { atomicExch(a.status, (int)KVMEM_E_DEVICE_RANGE); pg = 0; }
                return pg;                                    // a flagged id reads page 0; the status word reports it
            };
            int b0 = walk.t0 * boxes, page = lookup(b0 + lane), page_next = lookup(b0 + 32 + lane);
            const int z_view = walk.s * LG + walk.lg, row_tail = walk.s * a.tail_cap;
            for (int t = walk.t0; t < walk.t1; ++t, n += 2) {
                const bool in_view = t < walk.sp.view_tiles;
                const int tt = (t - walk.sp.view_tiles) * kTreeTile;      // first tail row of a tail tile
                const int live = in_view ? min(boxes, b_end - t * boxes) : min(2, (walk.sp.n_tail + walk.sp.n_q - tt + 63) / 64);
                if (PAGED && in_view && t * boxes >= b0 + 32) {
                    b0 += 32;
                    page = page_next;
                    page_next = lookup(b0 + 32 + lane);
                }
                // in a view tile of the pages the lane that looked a copy's page up issues it, else lanes 0 and 1
                const int u = PAGED && in_view ? b0 + lane - t * boxes : lane;
                const int st = n % RING;
                if (ok && n >= RING) ok = ptx::mbar_wait(&empty[st], (uint32_t)(((n / RING) & 1) ^ 1));
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) ptx::mbar_expect_tx(&full[st], (uint32_t)live * (uint32_t)(in_view ? box : 64) * 256u);
                __syncwarp();
                if (u >= 0 && u < live) {
                    unsigned char* dst = ring + (size_t)st * kTreeSlot + u * (in_view ? box : 64) * 128;
                    if (!in_view) {
                        ptx::tma_load_3d(dst, map_tail, 0, walk.lg, row_tail + tt + u * 64, &full[st]);
                        ptx::tma_load_3d(dst + kTreeHalf, map_tail, 64, walk.lg, row_tail + tt + u * 64, &full[st]);
                    } else {
                        // pages: [page][K | V][LG] tiles of B rows of 256 B
                        const int y = PAGED ? (per_block == 1 ? 0 : (b0 + lane) % per_block * 64) : t * kTreeTile + u * 64;
                        const int z = PAGED ? (page * 2 + kv) * LG + walk.lg : z_view;
                        ptx::tma_load_3d_hint(dst, map_in, 0, y, z, &full[st], once);
                        ptx::tma_load_3d_hint(dst + kTreeHalf, map_in, 64, y, z, &full[st], once);
                    }
                }
            }
            if (!ok) break;
        }
        // the copies still in flight land before the CTA gives its shared memory back
        for (int i = max(kv, n - RING); i < n; i += 2) ok = ptx::mbar_wait(&full[i % RING], (uint32_t)((i / RING) & 1)) && ok;
        if (!__all_sync(0xffffffffu, ok) && lane == 0) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
    } else if (warp == 1) {
        // ------------------------------------------------ MMA: one thread
        // Order: S(0) S(1) | O(0) S(2) | O(1) S(3) | ...: a slot's next logits are issued right behind the product that reads its
        // weights, in whose place they go.  MMAs that one thread issues run in order, so there is nothing to wait for.
        if (t5::elect()) {
            const uint32_t q_lo = t5::desc_lo(ptx::smem_u32(smem_q)), ring_lo = t5::desc_lo(ptx::smem_u32(ring));
            // Scalar code between the MMAs is latency: ring places move by addition, and the barriers of a step are asked together.
            struct Place {
                int st, ph;
                __device__ __forceinline__ void next() { st += 2; if (st >= RING) { st -= RING; ph ^= 1; } }
            } kp{0, 0}, vp{1, 0};                             // next key tile, next value tile
            int seg = 0, p_ph[2] = {0, 0};
            bool two = false;                                 // two row tiles: units are (tile, row tile), else tiles
            auto logits = [&](int x) {                        // S of slot x from the key tile at kp
                if (ok) {
                    t5::fence_after();
                    const uint32_t al = q_lo + (two ? (uint32_t)x * (kTreeSlot >> 4) : 0u), bl = ring_lo + (uint32_t)kp.st * (kTreeSlot >> 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t o = (uint32_t)(i >> 2) * (kTreeHalf >> 4) + (uint32_t)(i & 3) * 2u;
                        t5::mma_bf16(tmem + (uint32_t)x * 256u, t5::make_desc(al + o), t5::make_desc(bl + o), kTreeIdescS, i > 0 ? 1u : 0u);
                    }
                    t5::commit(&s_full[x]);
                    if (!two || x == 1) t5::commit(&empty[kp.st]);
                }
                if (!two || x == 1) kp.next();
            };
            while (walk.next<(QT == 2)>(a, w.row_groups)) {
                two = QT == 2 && walk.qt == 2;
                const int units = (walk.t1 - walk.t0) * (two ? 2 : 1);
                if (ok) ok = ptx::mbar_wait(&sh.q_full, (uint32_t)(seg & 1)) && ptx::mbar_wait(&full[kp.st], (uint32_t)kp.ph);
                logits(0);
                if (units > 1) {
                    if (ok && !two) ok = ptx::mbar_wait(&full[kp.st], (uint32_t)kp.ph);
                    logits(1);
                }
                for (int u = 0; u < units; ++u) {
                    const int x = u & 1;
                    const bool more = u + 2 < units, fresh = !two || x == 0;           // fresh: this slot meets the tiles first
                    if (ok) ok = ptx::mbar_wait_joint(fresh ? &full[vp.st] : nullptr, vp.ph, more && fresh ? &full[kp.st] : nullptr, kp.ph, &p_full[x], p_ph[x]);
                    p_ph[x] ^= 1;
                    if (ok) {
                        t5::fence_after();
                        const uint32_t bl = (ring_lo + (uint32_t)vp.st * (kTreeSlot >> 4)) | (kTreeVStep << 16);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            t5::mma_bf16_ta(tmem + (uint32_t)x * 256u + 128u, tmem + (uint32_t)x * 256u + (uint32_t)((i >> 2) * 64 + (i & 3) * 8),
                                            t5::make_desc(bl + (uint32_t)i * (2048u >> 4)), kTreeIdescO, u > 1 || i > 0 ? 1u : 0u);
                        if (!more) t5::commit(&o_done[x]);
                        if (!two || x == 1) t5::commit(&empty[vp.st]);
                    }
                    if (!two || x == 1) vp.next();
                    if (more) logits(x);
                }
                ++seg;
            }
            t5::commit(&sh.drained);                             // MMAs in flight end before the tensor memory is given back
            ok = ptx::mbar_wait(&sh.drained, 0u) && ok;
            if (!ok) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
        }
    } else {
        // ------------------------------------------------ rows: two threads a row, each with half of a tile's columns
        // Warps 2 .. 17: TMEM lanes 32 (warp & 3) + lane; groups of four warps are slot 0 columns 0 - 63, 64 - 127, slot 1 likewise.
        const int group = (warp - 2) >> 2, x = group >> 1, hh = group & 1, gt = (tid - 64) & 255;      // gt: thread of the slot's 256
        const int row_in = (warp & 3) * 32 + lane;                           // row of the row tile
        const uint32_t lanes = tmem + (uint32_t)x * 256u + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_addr = lanes + 64u * hh, o_addr = lanes + 128u + 64u * hh;
        const float scale2 = a.scale * 1.4426950408889634f;
        int tiles = 0, cnt = 0, done = 0;                   // tiles before this segment; units and finished segments of the slot
        auto wait = [&](uint64_t* bar, int phase) {
            if (ok) ok = ptx::mbar_wait(bar, (uint32_t)(phase & 1));
            ok = __all_sync(0xffffffffu, ok);
        };
        // the two warps that share the slot's rows 32 (warp & 3) ..
        auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(2 + x * 4 + (warp & 3)) : "memory"); };
        while (walk.next<(QT == 2)>(a, w.row_groups)) {
            const TreeSpan sp = walk.sp;
            const int l = walk.lg / a.G, g = walk.lg % a.G;
            const int rows = sp.n_q * a.r, row0 = walk.rg * 2 * kTreeRows;    // live rows of the head; the group's first
            const bool two = QT == 2 && walk.qt == 2;
            {
                // Q: all loads first, then, once both slots are done with the last segment's, the stores
                uint4 val[4 * QT];
                const int c = tid & 15;
#pragma unroll
                for (int i = 0; i < 4 * QT; ++i) {
                    const int row = row0 + ((tid - 64) >> 4) + 32 * i;
                    val[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (row < rows)
                        val[i] = *reinterpret_cast<const uint4*>(a.q + ((((size_t)walk.s * a.M + row / a.r) * a.L + l) * a.H + (size_t)g * a.r + row % a.r) * kTreeD + c * 8);
                }
                asm volatile("bar.sync 1, 512;" ::: "memory");
#pragma unroll
                for (int i = 0; i < 4 * QT; ++i) {
                    const int rr = ((tid - 64) >> 4) + 32 * i;
                    *reinterpret_cast<uint4*>(smem_q + (size_t)(rr >> 7) * kTreeSlot + (size_t)(c >> 3) * kTreeHalf + (rr & 127) * 128 + (((c & 7) ^ (rr & 7)) << 4)) = val[i];
                }
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.q_full);
            }
            const int row = row0 + (two ? x * kTreeRows : 0) + row_in;
            const bool warp_live = row - lane < rows;                         // any row of this warp is real
            const unsigned long long bits = row < rows ? tree_bits(a, walk.s, row / a.r, sp.n_q) : 0ull;
            float ref = -INFINITY, sum = 0.0f;
            bool cleared = false;
            const int n_units = two ? walk.t1 - walk.t0 : (walk.t1 - walk.t0 + 1 - x) >> 1;
            for (int j = 0; j < n_units; ++j) {
                const int ti = two ? j : 2 * j + x, t = walk.t0 + ti;
                const bool in_view = t < sp.view_tiles;
                const int c0 = (in_view ? t : t - sp.view_tiles) * kTreeTile;             // first token of the tile in view or tail
                const int n_valid = min(kTreeTile, (in_view ? sp.n_view : sp.n_tail + sp.n_q) - c0);
                const bool masked = n_valid < kTreeTile || (!in_view && c0 + kTreeTile > sp.n_tail);      // any column that some row does not see
                wait(&s_full[x], cnt);
                if (masked && (!two || x == 0)) {
                    // Values nobody sees become zero; drafted values that are not finite too (the merge adds them).  Only now: the tile
                    // that was in this ring slot before has landed for certain once these logits are there, and a wait for a phase
                    // two ahead of the barrier's would be over at once.
                    const int v = 2 * (tiles + ti) + 1, st = v % RING;
                    wait(&full[st], v / RING);
                    unsigned char* vt = ring + (size_t)st * kTreeSlot;
                    const int first = in_view ? n_valid : min(max(sp.n_tail - c0, 0), n_valid);
                    for (int i = first * 16 + gt; i < kTreeTile * 16; i += 256) {
                        const int rr = i >> 4, c = i & 15;
                        uint4* p = reinterpret_cast<uint4*>(vt + (size_t)(c >> 3) * kTreeHalf + rr * 128 + (((c & 7) ^ (rr & 7)) << 4));
                        uint4 val = make_uint4(0u, 0u, 0u, 0u);
                        bool put = true;
                        if (rr < n_valid) {
                            val = *p;
                            put = false;
                            uint32_t* e = reinterpret_cast<uint32_t*>(&val);
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                if ((e[h] & 0x00007f80u) == 0x00007f80u) { e[h] &= 0xffff0000u; put = true; }
                                if ((e[h] & 0x7f800000u) == 0x7f800000u) { e[h] &= 0x0000ffffu; put = true; }
                            }
                            cleared |= put;
                        }
                        if (put) *p = val;
                    }
                    ptx::fence_proxy_async_smem();
                }
                if (warp_live) {
                    t5::fence_after();
                    // Two sweeps over the thread's 64 logits, 32 at a time: the maximum, then the weights.  (All 64 held in between cost
                    // registers that spill, and a spill is slow here: shared memory leaves the L1 no room for it.)
                    uint32_t word0 = 0xffffffffu, word1 = 0xffffffffu;        // visible columns, 32 each
                    if (masked) {
                        auto word = [&](int c) {
                            const int left = n_valid - 64 * hh - 32 * c;
                            return in_view ? (left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u) : tail_word(c0 + 64 * hh + 32 * c, sp.n_tail, bits);
                        };
                        word0 = word(0);
                        word1 = word(1);
                    }
                    auto logits = [&](int c, uint32_t (&sv)[32]) {
                        t5::ld32_issue(s_addr + 32u * c, sv);
                        t5::ld_wait(sv);
                        if (masked) {
                            const uint32_t word = c == 0 ? word0 : word1;
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!((word >> i) & 1u)) sv[i] = 0xff800000u;
                        }
                    };
                    // (Loops, not unrolled: the first pass through fresh code costs more than the loops do.)
                    float m2 = -INFINITY;                         // the row's largest logit in this tile, NaN if one is
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        uint32_t sv[32];
                        logits(c, sv);
                        if (MASS && in_view && row < rows) {
                            float* lp = w.logits + (((size_t)walk.s * LG + walk.lg) * a.rows + row) * a.cap + c0 + 64 * hh + 32 * c;
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                if (64 * hh + 32 * c + i < n_valid)
                                    *reinterpret_cast<float4*>(lp + i) =
                                        make_float4(__uint_as_float(sv[i]) * scale2, __uint_as_float(sv[i + 1]) * scale2,
                                                    __uint_as_float(sv[i + 2]) * scale2, __uint_as_float(sv[i + 3]) * scale2);
                        }
                        float m[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t* e = &sv[i * 8];
                            m[i] = f2::max3_nan(f2::max3_nan(__uint_as_float(e[0]), __uint_as_float(e[1]), __uint_as_float(e[2])),
                                                f2::max3_nan(__uint_as_float(e[3]), __uint_as_float(e[4]), __uint_as_float(e[5])),
                                                f2::max3_nan(__uint_as_float(e[6]), __uint_as_float(e[7]), __uint_as_float(e[7])));
                        }
                        m2 = f2::max3_nan(f2::max3_nan(m[0], m[1], m[2]), m[3], m2);
                    }
                    sh.half_max[x][hh][row_in] = m2;
                    pair_sync();
                    m2 = scale2 * f2::max3_nan(m2, sh.half_max[x][hh ^ 1][row_in], m2);
                    // true for the first logit that is not -inf (ref is), and for a NaN
                    const bool moves = !(m2 <= ref + kTreeSlack) && m2 != -INFINITY;
                    if (__any_sync(0xffffffffu, moves)) {
                        const float to = moves ? m2 : ref, corr = moves ? t5::ex2(ref - to) : 1.0f;
                        if (j > 0) {
                            // the last product into O is complete: this tile's logits were issued after it
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
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
                    const bool unseen = ref == -INFINITY;         // nothing seen yet: every weight is exp2(-inf) = 0
                    const float use = unseen ? 0.0f : ref;
                    const uint64_t sc2 = f2::pk(scale2, scale2), nm2 = f2::pk(-use, -use);
                    uint64_t acc0 = f2::pk(0.0f, 0.0f), acc1 = acc0;
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        uint32_t sv[32], pk[16];
                        logits(c, sv);
                        tree_weights(sv, sc2, nm2, acc0, acc1, pk);
                        t5::st16(s_addr + 16u * c, pk);           // over logits that this thread has read
                    }
                    float a0, a1, a2, a3;
                    f2::unpk(acc0, a0, a1);
                    f2::unpk(acc1, a2, a3);
                    sum += (a0 + a1) + (a2 + a3);
                    t5::st_wait();
                    t5::fence_before();
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&p_full[x]);
                ++cnt;
            }
            // the segment's sums
            const size_t seg = (size_t)blockIdx.x + walk.head;
            if (n_units > 0) wait(&o_done[x], done++);
            if (warp_live) {
                t5::fence_after();
                const size_t at = (seg * 2 + x) * w.rows_slot + row_in;
                if (n_units > 0) {
                    // 16 columns at a time through 2 KB of this warp in the Q tiles, which no MMA reads any more, so that four
                    // lanes write 64 consecutive bytes of a row (a lane with 16 bytes of a row of its own takes four times as
                    // many cycles of the store path)
                    float4* stage = reinterpret_cast<float4*>(smem_q + (warp - 2) * 2048);
                    const int n_live = min(32, rows - (row - lane));
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t ov[16];
                        t5::ld16_issue(o_addr + 16u * c, ov);
                        t5::ld_wait(ov);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            stage[lane * 4 + (i ^ ((lane >> 1) & 3))] = make_float4(__uint_as_float(ov[4 * i]), __uint_as_float(ov[4 * i + 1]),
                                                                                     __uint_as_float(ov[4 * i + 2]), __uint_as_float(ov[4 * i + 3]));
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int rr = i * 8 + (lane >> 2);
                            if (rr < n_live)
                                *reinterpret_cast<float4*>(w.part_o + (at - lane + rr) * kTreeD + 64 * hh + 16 * c + 4 * (lane & 3)) =
                                    stage[rr * 4 + ((lane & 3) ^ ((rr >> 1) & 3))];
                        }
                        __syncwarp();
                    }
                }
                if (hh == 1) sh.half_max[x][1][row_in] = sum;
                pair_sync();
                if (hh == 0 && row < rows) w.part_ml[at] = make_float2(ref, sum + sh.half_max[x][1][row_in]);
                t5::fence_before();
            }
            cleared = __any_sync(0xffffffffu, cleared);
            if (lane == 0) reinterpret_cast<unsigned char*>(w.part_nf + seg)[warp - 2] = cleared ? 1 : 0;
            tiles += walk.t1 - walk.t0;
        }
        if (!ok && lane == 0) atomicExch(a.status, (int)KVMEM_E_TIMEOUT);
    }
    t5::fence_before();
    __syncthreads();
    if (warp == 1) {
        t5::fence_after();
        t5::tmem_dealloc(tmem, 512);
    }
}

// Joins the segments of one query row in the order of the line, four dimensions a lane.  Bound by latency (a round of dependent
// reads costs some 2 us here), so a row gets WARPS warps, each with a run of its shares, as far as all rows are then resident
// at a time (one CTA an SM), and a warp requests sixteen sums together.  Four warps against one, a call at 2,048 tokens and 32
// rows per KV head: 13.7 us against 15.7; at 2,048 rows in all the merge alone takes 28 us with four and 7.6 with one.
constexpr int kMergeThreads = 256;
template <int WARPS>
__global__ void __launch_bounds__(kMergeThreads, WARPS == 1 ? 2 : 1)
tree_merge_kernel(const __grid_constant__ TreeWork w) {
    constexpr int ROWS = kMergeThreads / 32 / WARPS;
    __shared__ float4 sums[ROWS][WARPS][32];
    __shared__ float2 stats[ROWS][WARPS];
    pdl_wait();
    pdl_trigger();
    const TreeArgs& a = w.a;
    const int LG = a.L * a.G, hz = blockIdx.x, s = hz / LG, lg = hz % LG, lane = threadIdx.x & 31;
    const int part = (threadIdx.x >> 5) % WARPS, mine = (threadIdx.x >> 5) / WARPS;
    const int row = blockIdx.y * ROWS + mine;
    const TreeInfo in = w.info[s], line = w.info[a.ns];
    const int m = row / a.r;
    const bool there = m < in.n_q;
    float z = 0.0f, top = -INFINITY;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    bool nf = false;
    if (there && in.tiles > 0) {
        const int rg = row / (2 * kTreeRows), rr = row % (2 * kTreeRows);
        int first = in.start + lg * (in.tiles + line.groups) + line.groups, shift = 0;
        if (a.rows > kTreeRows) {
            const TreeCosts u(TreeSpan{0, 0, in.n_q, 0, in.tiles, in.groups}, a.r, line.groups);
            first = in.start + lg * u.head + rg * u.full + line.groups;
            shift = rg == in.groups - 1 ? u.shift : 1;
        }
        const int last_tile = first + ((in.tiles - 1) << shift);
        const int c0 = line_owner(first, line.start, line.tiles), c1 = line_owner(last_tile, line.start, line.tiles);
        const size_t seg = ((size_t)s * LG + lg) * w.row_groups + rg + c0;
        // one row tile: both slots hold a share of every row; two: slot rr / 128 does
        const int per = tree_row_tiles(in.n_q * a.r, rg) == 1 ? 2 : 1, parts = (c1 - c0 + 1) * per;
        const size_t at0 = (seg * 2 + (per == 1 ? rr >> 7 : 0)) * w.rows_slot + (rr & 127), step = (size_t)(3 - per) * w.rows_slot;
        const float4* po = reinterpret_cast<const float4*>(w.part_o + at0 * kTreeD) + lane;
        for (int c = lane; c <= c1 - c0; c += 32) { const ulonglong2 f = w.part_nf[seg + c]; nf |= (f.x | f.y) != 0; }
        // the statistics of 32 shares at a time, a lane each; what there is is rescaled when the maximum grows
        const int last = (int)((long long)parts * (part + 1) / WARPS);
        for (int i0 = (int)((long long)parts * part / WARPS); i0 < last; i0 += 32) {
            const int left = min(32, last - i0);
            const float2 ml = lane < left ? w.part_ml[at0 + (size_t)(i0 + lane) * step] : make_float2(-INFINITY, 0.0f);
            const bool holds = ml.x > -INFINITY || ml.y != 0.0f;          // a share without a visible token holds no sums
            const uint32_t live = __ballot_sync(0xffffffffu, holds);
            float mx = ml.x;
#pragma unroll
            for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float to = fmaxf(top, mx), back = top > -INFINITY ? t5::ex2(top - to) : 1.0f;
            const float f = holds ? t5::ex2(ml.x - to) : 0.0f;
            float zi = holds ? f * ml.y : 0.0f;
#pragma unroll
            for (int d = 16; d; d >>= 1) zi += __shfl_xor_sync(0xffffffffu, zi, d);
            acc.x *= back; acc.y *= back; acc.z *= back; acc.w *= back;
            z = z * back + zi;
            top = to;
#pragma unroll 1
            for (int u0 = 0; u0 < left; u0 += 16) {
                float4 v[16];
#pragma unroll
                for (int u = 0; u < 16; ++u)
                    if ((live >> (u0 + u)) & 1u) v[u] = po[(size_t)(i0 + u0 + u) * step * (kTreeD / 4)];
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const float fu = __shfl_sync(0xffffffffu, f, u0 + u);
                    if ((live >> (u0 + u)) & 1u) { acc.x += fu * v[u].x; acc.y += fu * v[u].y; acc.z += fu * v[u].z; acc.w += fu * v[u].w; }
                }
            }
        }
        nf = __any_sync(0xffffffffu, nf);
    }
    if (WARPS > 1) {
        sums[mine][part][lane] = acc;
        if (lane == 0) stats[mine][part] = make_float2(top, z);
        __syncthreads();
    }
    if (part > 0 || !there) return;
    if (WARPS > 1) {
#pragma unroll
        for (int i = 0; i < WARPS; ++i) top = fmaxf(top, stats[mine][i].x);
        z = 0.0f;
        acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const float2 st = stats[mine][i];
            if (st.x > -INFINITY || st.y != 0.0f) {
                const float f = t5::ex2(st.x - top);
                const float4 v = sums[mine][i][lane];
                z += f * st.y;
                acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            }
        }
    }
    const size_t orow = (((size_t)s * a.M + m) * a.L + lg / a.G) * a.H + (size_t)(lg % a.G) * a.r + row % a.r;
    const bool none = z == 0.0f;
    float out[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!none) { out[0] = acc.x / z; out[1] = acc.y / z; out[2] = acc.z / z; out[3] = acc.w / z; }
    if (nf && !none) {
        // drafted values that are not finite were left out: they reach the rows that see them here
        const unsigned long long bits = tree_bits(a, s, m, in.n_q);
        for (int j = 0; j < in.n_q; ++j)
            if ((bits >> j) & 1) {
                const __nv_bfloat16* vr = a.tail_v + (((size_t)s * a.tail_cap + in.n_tail + j) * LG + lg) * kTreeD + 4 * lane;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = __bfloat162float(vr[i]);
                    if (!isfinite(v)) out[i] += v;
                }
            }
    }
    *reinterpret_cast<uint2*>(a.out + orow * kTreeD + 4 * lane) = make_uint2(ptx::pack_bf16x2(out[0], out[1]), ptx::pack_bf16x2(out[2], out[3]));
    const float lse2 = none ? -INFINITY : top + log2f(z);
    if (lane == 0) {
        a.lse[orow] = lse2 * 0.6931471805599453f;
        // a row without any weight adds none to its tokens: exp2(x - inf) = 0 there, where -inf - -inf would be NaN
        if (w.lse2) w.lse2[(size_t)hz * a.rows + row] = none ? INFINITY : lse2;
    }
}

// mass = decay mass + sum over the rows of exp2(logit - lse), from the logits that the attention left.  A warp takes 256 tokens,
// eight a lane, and four to eight of the rows, so that a thread has eight loads in flight; `split` warps (1, 2, 4, 8) share out
// the rows of their tokens and a block's warps cover WARPS / split runs of tokens.  Whole calls (attention, merge, weights) with
// 1, 2, 4, 8 warps to a row set, in us: 64 heads of 10,240 tokens 64.6, 65.3, 65.7, 68.6 at one row, 69.5, 67.9, 67.9, 70.6 at 4,
// 72.1, 69.3, 69.2, 71.3 at 8, 79.8, 76.0, 74.3, 76.2 at 16, 115, 106, 102, 104 at 32, 214, 187, 176, 177 at 64; 8 heads of 262,144
// tokens 184, 184, 187, 193 at 4 rows, 202, 199, 200, 207 at 8, 239, 231, 231, 237 at 16, 308, 298, 296, 300 at 32, 541, 503, 492,
// 500 at 64.
constexpr int kMassTokens = 256;
template <int split, int WARPS>
__global__ void __launch_bounds__(32 * WARPS)
tree_mass_kernel(const __grid_constant__ TreeWork w) {
    __shared__ float4 sums[WARPS][2][32];
    pdl_wait();
    pdl_trigger();
    const TreeArgs& a = w.a;
    const int hz = blockIdx.x, s = hz / (a.L * a.G), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const TreeSpan sp = tree_span(a, s, false);
    const int block0 = blockIdx.y * (kMassTokens * (WARPS / split));
    if (block0 >= sp.n_view) return;
    const int rows = sp.n_q * a.r, part = warp % split, t0 = block0 + warp / split * kMassTokens + 4 * lane;
    float4* mp = reinterpret_cast<float4*>(a.mass + (size_t)hz * a.cap + t0);
    float4 sum[2], m[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        sum[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (part == 0 && t0 + 128 * e < sp.n_view) m[e] = mp[32 * e];       // n_view is a multiple of 16
    }
#pragma unroll 4
    for (int row = part; row < rows; row += split) {
        const float4* lp = reinterpret_cast<const float4*>(w.logits + ((size_t)hz * a.rows + row) * a.cap + t0);
        const float z = w.lse2[(size_t)hz * a.rows + row];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (t0 + 128 * e < sp.n_view) {
                const float4 v = __ldcs(lp + 32 * e);
                sum[e].x += t5::ex2(v.x - z); sum[e].y += t5::ex2(v.y - z); sum[e].z += t5::ex2(v.z - z); sum[e].w += t5::ex2(v.w - z);
            }
    }
    if (split > 1) {
#pragma unroll
        for (int e = 0; e < 2; ++e) sums[warp][e][lane] = sum[e];
        __syncthreads();
        if (part > 0) return;
        for (int i = 1; i < split; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float4 v = sums[warp + i][e][lane];
                sum[e].x += v.x; sum[e].y += v.y; sum[e].z += v.z; sum[e].w += v.w;
            }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (t0 + 128 * e < sp.n_view)
            mp[32 * e] = make_float4(fmaf(a.decay, m[e].x, sum[e].x), fmaf(a.decay, m[e].y, sum[e].y), fmaf(a.decay, m[e].z, sum[e].z), fmaf(a.decay, m[e].w, sum[e].w));
}

// sizes and places inside the workspace; base null: sizes alone
static size_t plan_tree(const kvmem_pool_config_t& c, int n_sessions, int M, int mass_cap, char* base, TreeWork* w) {
    const int rows = M * (c.n_q_heads / c.n_kv_heads);
    w->row_groups = (rows + 2 * kTreeRows - 1) / (2 * kTreeRows);
    w->rows_slot = std::min(rows, kTreeRows);
    const size_t heads = (size_t)n_sessions * c.n_layers * c.n_kv_heads, segs = heads * w->row_groups + kSMs;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return base ? base + at : nullptr; };
    w->part_o = (float*)take(segs * 2 * w->rows_slot * kTreeD * sizeof(float));
    w->part_ml = (float2*)take(segs * 2 * w->rows_slot * sizeof(float2));
    w->part_nf = (ulonglong2*)take(segs * sizeof(ulonglong2));
    w->info = (TreeInfo*)take(((size_t)n_sessions + 1) * sizeof(TreeInfo));
    w->lse2 = mass_cap ? (float*)take(heads * rows * sizeof(float)) : nullptr;
    w->logits = mass_cap ? (float*)take(heads * rows * mass_cap * sizeof(float)) : nullptr;
    return off;
}

size_t tree_workspace_bytes(const kvmem_pool_config_t& c, int n_sessions, int n_q_tokens, int mass_cap_tokens) {
    TreeWork w;
    return plan_tree(c, n_sessions, n_q_tokens, mass_cap_tokens, nullptr, &w);
}

// most tiles of a row group, counted from the capacities
static long long tree_tiles(int cap, int tail_cap) { return ((long long)cap + kTreeTile - 1) / kTreeTile + ((long long)tail_cap + kTreeTile - 1) / kTreeTile; }

bool tree_line_fits(const kvmem_pool_config_t& c, int n_sessions, int n_q_tokens, int cap_tokens, int tail_cap_tokens) {
    const long long rows = (long long)n_q_tokens * (c.n_q_heads / c.n_kv_heads);
    const long long groups = (long long)n_sessions * c.n_layers * c.n_kv_heads * ((rows + 2 * kTreeRows - 1) / (2 * kTreeRows));
    const bool wide = rows > kTreeRows;
    return groups < kTreeMostUnits && groups * (tree_tiles(cap_tokens, tail_cap_tokens) * tree_most(wide) + tree_lead(wide)) < kTreeMostUnits;
}

// [outer][rows][128 dims] bf16, boxes of 64 dims x box_rows x 1, 128-byte swizzle; tail: [tokens][heads][128] with boxes of 64 tokens
static bool tree_map(CUtensorMap* map, const __nv_bfloat16* p, cuuint64_t d1, cuuint64_t d2, cuuint32_t box1, cuuint32_t box2) {
    static PFN_cuTensorMapEncodeTiled_v12000 enc = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr) : nullptr;
    }();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)kTreeD, d1, d2};
    cuuint64_t strides[2] = {(cuuint64_t)kTreeD * 2, d1 * kTreeD * 2};
    cuuint32_t box[3] = {64, box1, box2}, step[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int QT, bool PAGED, bool MASS>
static cudaError_t launch_split(const kvmem_pool& p, int grid, cudaStream_t st, const CUtensorMap (&m)[4], const TreeWork& w) {
    static PerDeviceOnce done;
    if (done.pending(p.cfg.device)) {
        const cudaError_t e = cudaFuncSetAttribute(tree_split_kernel<QT, PAGED, MASS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tree_smem(QT));
        if (e != cudaSuccess) return e;
        done.mark(p.cfg.device);
    }
    return launch_pdl(tree_split_kernel<QT, PAGED, MASS>, dim3((unsigned)grid), dim3(kTreeThreads), tree_smem(QT), st, m[0], m[1], m[2], m[3], w);
}

cudaError_t launch_tree(const kvmem_pool& p, const TreeArgs& a, void* workspace, cudaStream_t st) {
    const int LG = a.L * a.G;
    TreeWork w{};
    plan_tree(p.cfg, a.ns, a.M, a.mass ? a.cap : 0, (char*)workspace, &w);
    w.a = a;
    CUtensorMap m[4];
    const bool paged = a.view_k == nullptr;
    bool made = paged ? tree_map(&m[0], a.pages, (cuuint64_t)a.B, (cuuint64_t)a.max_blocks * 2 * LG, (cuuint32_t)std::min(a.B, 64), 1)
                      : tree_map(&m[0], a.view_k, (cuuint64_t)a.cap, (cuuint64_t)a.ns * LG, 64, 1) &&
                            tree_map(&m[1], a.view_v, (cuuint64_t)a.cap, (cuuint64_t)a.ns * LG, 64, 1);
    if (paged) m[1] = m[0];
    if (a.tail_k)
        made = made && tree_map(&m[2], a.tail_k, (cuuint64_t)LG, (cuuint64_t)a.ns * a.tail_cap, 1, 64) &&
               tree_map(&m[3], a.tail_v, (cuuint64_t)LG, (cuuint64_t)a.ns * a.tail_cap, 1, 64);
    else m[2] = m[3] = m[0];
    if (!made) return cudaErrorInvalidValue;
    const int grid = (int)std::min<long long>(std::min(p.sm_count, kSMs), (long long)a.ns * LG * w.row_groups * tree_tiles(a.cap, a.tail_cap));
    cudaError_t e;
    if (a.mass) e = launch_split<1, false, true>(p, grid, st, m, w);            // at most 64 rows
    else if (paged) e = a.rows <= kTreeRows ? launch_split<1, true, false>(p, grid, st, m, w) : launch_split<2, true, false>(p, grid, st, m, w);
    else e = a.rows <= kTreeRows ? launch_split<1, false, false>(p, grid, st, m, w) : launch_split<2, false, false>(p, grid, st, m, w);
    if (e != cudaSuccess) return e;
    const long long all_rows = (long long)a.ns * LG * a.rows;
    auto merge = [&](auto kernel, int rows) {
        return launch_pdl(kernel, dim3((unsigned)(a.ns * LG), (unsigned)((a.rows + rows - 1) / rows)), dim3(kMergeThreads), 0, st, w);
    };
    e = all_rows <= kSMs ? merge(tree_merge_kernel<8>, 1) : all_rows <= 2 * kSMs ? merge(tree_merge_kernel<4>, 2)
      : all_rows <= 4 * kSMs ? merge(tree_merge_kernel<2>, 4) : merge(tree_merge_kernel<1>, 8);
    if (e != cudaSuccess || !a.mass) return e;
    auto weights = [&](auto kernel, int tokens, int warps) {
        return launch_pdl(kernel, dim3((unsigned)(a.ns * LG), (unsigned)((a.cap + tokens - 1) / tokens)), dim3(32 * warps), 0, st, w);
    };
    // Few rows and enough tokens to fill the SMs in long runs: whole warps on tokens; else the rows are shared out (5.3 -> 3.3 us at
    // 2,048 tokens).  The two sides are within 3 % of one another where they meet.
    const bool many = (long long)a.ns * LG * (a.cap / (8 * kMassTokens)) >= 2 * kSMs;
    return many && a.rows <= 4 ? weights(tree_mass_kernel<1, 8>, 8 * kMassTokens, 8) : many && a.rows <= 8 ? weights(tree_mass_kernel<2, 8>, 4 * kMassTokens, 8)
         : a.rows <= 16 ? weights(tree_mass_kernel<4, 4>, kMassTokens, 4) : weights(tree_mass_kernel<8, 8>, kMassTokens, 8);
}

}  // namespace kvmem
