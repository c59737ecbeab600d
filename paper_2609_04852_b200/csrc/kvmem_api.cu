// C ABI of libkvmem_b200: argument checking, pool and session bookkeeping, launch sequencing.
// Every step of the recall path runs in the kernels of the sibling files; nothing here computes.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <thread>

#include "kvmem_internal.cuh"

namespace kvmem {

static thread_local char g_err[512] = "";

void set_error(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
}

bool config_valid(const kvmem_pool_config_t& c, const char** why) {
    auto bad = [&](const char* w) { *why = w; return false; };
    if (c.n_layers < 1 || c.n_layers > 256) return bad("n_layers must be in [1, 256]");
    if (c.n_kv_heads < 1 || c.n_q_heads < 1 || c.n_q_heads % c.n_kv_heads != 0)
        return bad("n_q_heads must be a positive multiple of n_kv_heads");
    if (c.head_dim < 8 || c.head_dim > 512 || c.head_dim % 8 != 0) return bad("head_dim must be a multiple of 8 in [8, 512]");
    if (c.block_tokens < 16 || c.block_tokens > 256 || c.block_tokens % 16 != 0)
        return bad("block_tokens must be a multiple of 16 in [16, 256]");
    if (c.max_sessions < 1 || c.max_sessions > 65535) return bad("max_sessions must be in [1, 65535]");
    if (c.max_blocks < 1) return bad("max_blocks must be positive");
    if (c.max_blocks_per_session < 1 || c.max_blocks_per_session > c.max_blocks)
        return bad("max_blocks_per_session must be in [1, max_blocks]");
    if (c.device < 0) return bad("device must be a CUDA ordinal");
    if (c.rope_max_positions < 0) return bad("rope_max_positions must be non-negative");
    if (c.rope_max_positions > 0 && !(c.rope_theta > 1.0f)) return bad("rope_theta must exceed 1 when rotary support is on");
    if (c.rope_max_positions > 0 && c.head_dim % 16 != 0) return bad("rotary support needs head_dim to be a multiple of 16");
    if (c.rope_in_block_keys != 0 && c.rope_in_block_keys != 1) return bad("rope_in_block_keys must be 0 or 1");
    if (c.rope_in_block_keys && c.rope_max_positions < c.block_tokens)
        return bad("rope_in_block_keys needs rotary support covering at least one block (rope_max_positions >= block_tokens)");
    if (c.fp8_pages != 0 && c.fp8_pages != 1) return bad("fp8_pages must be 0 or 1");
    if (c.fp8_pages) {
        if (c.head_dim != 128 || c.block_tokens != 64) return bad("an FP8 repository needs head_dim 128 and 64-token blocks");
        if (c.rope_max_positions > 0 && !c.rope_in_block_keys)
            return bad("an FP8 repository with rotary support needs rope_in_block_keys (codes cannot be re-encoded; the query is rotated instead)");
        if (!(c.fp8_k_scale > 0.0f) || !(c.fp8_v_scale > 0.0f) || !std::isfinite(c.fp8_k_scale) || !std::isfinite(c.fp8_v_scale))
            return bad("fp8_k_scale and fp8_v_scale must be positive and finite");
    }
    return true;
}

Layout make_layout(const kvmem_pool_config_t& c) {
    Layout l{};
    l.tile_elems = (size_t)c.block_tokens * c.head_dim;
    l.page_elems = 2 * (size_t)c.n_layers * c.n_kv_heads * l.tile_elems;
    l.index_elems_per_session = (size_t)c.n_layers * c.n_kv_heads * c.max_blocks_per_session * c.head_dim;
    size_t off = 0;
    l.pages_off = off;
    off = align_up(off + (size_t)c.max_blocks * l.page_elems * (c.fp8_pages ? 1 : 2), 256);      // bf16 or E4M3 elements
    l.index_off = off;
    off = align_up(off + (size_t)c.max_sessions * l.index_elems_per_session * 2, 256);
    l.tables_off = off;
    off = align_up(off + (size_t)c.max_sessions * c.max_blocks_per_session * 4, 256);
    l.nblocks_off = off;
    off = align_up(off + (size_t)c.max_sessions * 4, 256);
    l.status_off = off;
    off = align_up(off + 256, 256);
    l.pos0_off = off;
    if (c.rope_max_positions > 0) off = align_up(off + (size_t)c.max_sessions * c.max_blocks_per_session * 4, 256);
    l.rope_off = off;
    if (c.rope_max_positions > 0) off = align_up(off + (size_t)c.rope_max_positions * (c.head_dim / 2) * sizeof(float2), 256);
    l.total = off;
    return l;
}

static bool pool_ok(const kvmem_pool* p) {
    if (!p || p->magic != kMagic) {
        set_error("pool handle is null or stale");
        return false;
    }
    return true;
}

// pool_ok plus: the pool's device is the calling thread's current device.  Every call that enqueues work launches on the
// current device with the pool's pointers, so a mismatch is refused on the host instead of faulting on the wrong GPU.
static bool pool_live(const kvmem_pool* p) {
    if (!pool_ok(p)) return false;
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device != p->cfg.device) {
        (void)cudaGetLastError();
        set_error("the pool lives on device %d but device %d is current", p->cfg.device, device);
        return false;
    }
    return true;
}

static bool sessions_ok(const kvmem_pool* p, int first, int n) {
    if (first < 0 || n < 1 || first > p->cfg.max_sessions - n) {
        set_error("sessions [%d, %lld) outside [0, %d)", first, (long long)first + n, p->cfg.max_sessions);
        return false;
    }
    return true;
}

// the calls that read bf16 pages refuse an FP8 repository (and the other way round) instead of misreading it
static bool pages_are(const kvmem_pool* p, bool fp8, const char* who) {
    if ((p->cfg.fp8_pages != 0) == fp8) return true;
    set_error("%s reads %s pages, the pool holds %s", who, fp8 ? "FP8" : "bf16", fp8 ? "bf16" : "FP8");
    return false;
}

static int cuda_fail(const char* what, cudaError_t e) {
    set_error("%s: %s", what, cudaGetErrorString(e));
    return KVMEM_E_CUDA;
}

// f(begin, end) over [0, n), shared out over up to 16 host threads (a rotary table of 262,144 positions takes one of them 0.24 s); where no
// thread is to be had, on this one
template <typename F>
static void on_threads(int n, const F& f) {
    const int most = std::max(1, std::min({16, (int)std::thread::hardware_concurrency(), n / 256}));
    std::thread t[16];
    int started = 1;                       // pieces that have a thread; this one takes the first and what is left
    try {
        for (; started < most; ++started) {
            const int a = (int)((int64_t)n * started / most), b = (int)((int64_t)n * (started + 1) / most);
            t[started] = std::thread([&f, a, b] { f(a, b); });
        }
    } catch (...) {}
    f(0, (int)((int64_t)n / most));
    if (started < most) f((int)((int64_t)n * started / most), n);
    for (int i = 1; i < started; ++i) t[i].join();
}

// frequencies of the pool's own rotary form: theta^(-2i/d)
static void own_frequencies(const kvmem_pool_config_t& c, double* f) {
    for (int i = 0; i < c.head_dim / 2; ++i) f[i] = pow((double)c.rope_theta, -2.0 * (double)i / (double)c.head_dim);
}

// cos/sin of position * frequency in fp64, one rounding to fp32, computed here on the host; 8,192 positions at a time in one buffer, used
// again when its copy is over (whether a copy from pageable memory is staged or read later is the system's choice)
static int upload_rope_table(const kvmem_pool& p, const double* freq, cudaStream_t st) {
    const int half = p.cfg.head_dim / 2, positions = p.cfg.rope_max_positions, chunk = 8192;
    const std::unique_ptr<float2[]> rows(new (std::nothrow) float2[(size_t)std::min(chunk, positions) * half]);
    if (!rows) { set_error("host allocation failed"); return KVMEM_E_CAPACITY; }
    for (int p0 = 0; p0 < positions; p0 += chunk) {
        const int n = std::min(chunk, positions - p0);
        on_threads(n, [&](int r0, int r1) {
            for (int r = r0; r < r1; ++r)
                for (int i = 0; i < half; ++i) {
                    const double ang = (double)(p0 + r) * freq[i];
                    rows[(size_t)r * half + i] = make_float2((float)cos(ang), (float)sin(ang));
                }
        });
        cudaError_t e = cudaMemcpyAsync(p.rope_dev + (size_t)p0 * half, rows.get(), (size_t)n * half * sizeof(float2), cudaMemcpyHostToDevice, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
        if (e != cudaSuccess) return cuda_fail("rotary table upload", e);
    }
    return KVMEM_OK;
}

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// The passes that read pages through the block table walk the view in 64-token tiles: a tile is 64 / B whole blocks or
// a 64-token slice of one block.  in_block_rotation: the pass rotates by one angle set per tile (in-block key layout),
// which needs tile == block.
static bool paged_block_size_ok(const kvmem_pool* p, bool in_block_rotation, const char* who) {
    const int B = p->cfg.block_tokens;
    if (p->cfg.head_dim != 128 || !(64 % B == 0 || B % 64 == 0)) {
        set_error("%s is built for head_dim 128 and block sizes that divide or are a multiple of 64 tokens", who);
        return false;
    }
    if (in_block_rotation && B != 64) {
        set_error("%s on a pool with rope_in_block_keys rotates once per 64-token tile and needs 64-token blocks", who);
        return false;
    }
    return true;
}

}  // namespace kvmem

using namespace kvmem;

extern "C" {

const char* kvmem_last_error(void) { return g_err; }

size_t kvmem_pool_bytes(const kvmem_pool_config_t* cfg) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why)) {
        set_error("invalid pool configuration: %s", cfg ? why : "null");
        return 0;
    }
    return make_layout(*cfg).total;
}

int32_t kvmem_budget_blocks(const kvmem_select_params_t* prm, int32_t block_tokens, int32_t n_blocks) {
    if (!prm || block_tokens <= 0) return 0;
    int64_t room = (int64_t)prm->max_view_tokens - (int64_t)prm->mandatory_tokens;
    int64_t k = room > 0 ? room / block_tokens : 0;
    k = std::min<int64_t>(k, prm->budget_blocks);
    k = std::min<int64_t>(k, n_blocks);
    return (int32_t)std::max<int64_t>(k, 0);
}

size_t kvmem_select_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why) || n_sessions < 1 || n_sessions > cfg->max_sessions || n_q_tokens < 1) {
        set_error("invalid arguments to kvmem_select_workspace_bytes");
        return 0;
    }
    if (n_q_tokens > kMaxDecodeTokens) return plan_chunk_workspace(*cfg, n_sessions, n_q_tokens, nullptr).total;
    return plan_score_workspace(*cfg, n_sessions, n_q_tokens, nullptr).total;
}

size_t kvmem_attend_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why) || n_sessions < 1 || n_q_tokens < 1) {
        set_error("invalid arguments to kvmem_attend_workspace_bytes");
        return 0;
    }
    return plan_attend(*cfg, n_sessions, n_q_tokens, kSMs).total;
}

int kvmem_pool_create(const kvmem_pool_config_t* cfg, void* storage, size_t bytes, kvmem_pool_t** out) {
    const char* why = "";
    if (!out) { set_error("out is null"); return KVMEM_E_INVALID; }
    *out = nullptr;
    if (!cfg || !config_valid(*cfg, &why)) {
        set_error("invalid pool configuration: %s", cfg ? why : "null");
        return KVMEM_E_INVALID;
    }
    if (!storage || !aligned(storage, 256)) { set_error("storage must be a 256-byte aligned device pointer"); return KVMEM_E_INVALID; }
    Layout lay = make_layout(*cfg);
    if (bytes < lay.total) {
        set_error("storage holds %zu bytes, the pool needs %zu", bytes, lay.total);
        return KVMEM_E_CAPACITY;
    }
    cudaError_t e = cudaSetDevice(cfg->device);
    if (e != cudaSuccess) return cuda_fail("cudaSetDevice", e);
    cudaDeviceProp prop;
    e = cudaGetDeviceProperties(&prop, cfg->device);
    if (e != cudaSuccess) return cuda_fail("cudaGetDeviceProperties", e);
    if (prop.major != 10) {
        set_error("device %d is compute capability %d.%d; this library is built for sm_100a only", cfg->device,
                  prop.major, prop.minor);
        return KVMEM_E_UNSUPPORTED;
    }
    kvmem_pool* p = new (std::nothrow) kvmem_pool();
    if (!p) { set_error("host allocation failed"); return KVMEM_E_CAPACITY; }
    p->magic = kMagic;
    p->cfg = *cfg;
    p->geo = Geometry{cfg->n_layers, cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, cfg->block_tokens,
                      cfg->n_q_heads / cfg->n_kv_heads, cfg->max_sessions, cfg->max_blocks, cfg->max_blocks_per_session};
    p->lay = lay;
    p->base = (char*)storage;
    p->pages = (__nv_bfloat16*)(p->base + lay.pages_off);
    p->index = (__nv_bfloat16*)(p->base + lay.index_off);
    p->tables = (int32_t*)(p->base + lay.tables_off);
    p->nblocks_dev = (int32_t*)(p->base + lay.nblocks_off);
    p->status_dev = (int32_t*)(p->base + lay.status_off);
    p->sess_blocks.assign(cfg->max_sessions, 0);
    p->sess_pages.assign(cfg->max_sessions, {});
    p->sess_reserved.assign(cfg->max_sessions, {});
    p->rope_form = RopeForm{cfg->head_dim, cfg->head_dim / 16, 0};
    p->page_used.assign(cfg->max_blocks, 0);
    p->free_hint = 0;
    p->sm_count = prop.multiProcessorCount;
    p->pos0_dev = cfg->rope_max_positions > 0 ? (int32_t*)(p->base + lay.pos0_off) : nullptr;
    p->rope_dev = cfg->rope_max_positions > 0 ? (float2*)(p->base + lay.rope_off) : nullptr;
    e = cudaMemset(p->base + lay.tables_off, 0xff, lay.nblocks_off - lay.tables_off);
    if (e == cudaSuccess) e = cudaMemset(p->base + lay.nblocks_off, 0, lay.rope_off - lay.nblocks_off);
    if (e == cudaSuccess && cfg->rope_max_positions > 0) {
        double freq[256];
        own_frequencies(*cfg, freq);
        const int rc = upload_rope_table(*p, freq, nullptr);
        if (rc != KVMEM_OK) { (void)cudaDeviceSynchronize(); delete p; return rc; }
        p->rope_own = true;
    }
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) { delete p; return cuda_fail("clearing pool metadata", e); }
    *out = p;
    return KVMEM_OK;
}

int kvmem_pool_destroy(kvmem_pool_t* pool) {
    if (!pool_ok(pool)) return KVMEM_E_STATE;
    pool->magic = 0;
    if (pool->copy_stream) {            // the copy stream of host-resident index scoring: drain it, then let it go
        cudaStreamSynchronize(pool->copy_stream);
        for (int i = 0; i < 2; ++i) {
            if (pool->ev_ready[i]) cudaEventDestroy(pool->ev_ready[i]);
            if (pool->ev_free[i]) cudaEventDestroy(pool->ev_free[i]);
        }
        if (pool->ev_start) cudaEventDestroy(pool->ev_start);
        cudaStreamDestroy(pool->copy_stream);
    }
    delete pool;
    return KVMEM_OK;
}

int kvmem_session_reset(kvmem_pool_t* p, int32_t session, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    // the device's block count first: kernels that size their work from it see an empty session from here on in stream order
    cudaError_t e = cudaMemsetAsync(p->nblocks_dev + session, 0, 4, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("clearing the session's block count", e);
    // no entry of its table is a page from here on: what appends tokens to reserved blocks goes by that
    const size_t entries = p->sess_pages[session].size() + p->sess_reserved[session].size();
    if (entries) e = cudaMemsetAsync(p->tables + (size_t)session * p->cfg.max_blocks_per_session, 0xff, entries * 4, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("clearing the session's block table", e);
    for (int32_t pg : p->sess_pages[session]) p->page_used[pg] = 0;
    for (int32_t pg : p->sess_reserved[session]) p->page_used[pg] = 0;
    p->sess_pages[session].clear();
    p->sess_reserved[session].clear();
    p->sess_blocks[session] = 0;
    p->free_hint = 0;
    return KVMEM_OK;
}

int32_t kvmem_session_blocks(const kvmem_pool_t* p, int32_t session) {
    if (!pool_ok(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    return p->sess_blocks[session];
}

// n_blocks free pages, the caller's or the lowest, without touching the pool
static int choose_pages(const kvmem_pool* p, int32_t n_blocks, const int32_t* phys_ids, std::vector<int32_t>& ids) {
    if (phys_ids) {
        std::vector<int32_t> sorted(phys_ids, phys_ids + n_blocks);
        std::sort(sorted.begin(), sorted.end());
        for (int i = 0; i < n_blocks; ++i) {
            int32_t pg = phys_ids[i];
            if (pg < 0 || pg >= p->cfg.max_blocks) { set_error("page id %d outside [0, %d)", pg, p->cfg.max_blocks); return KVMEM_E_INVALID; }
            if (p->page_used[pg]) { set_error("page %d is already in use", pg); return KVMEM_E_STATE; }
            if (i > 0 && sorted[i] == sorted[i - 1]) { set_error("page id %d given twice", sorted[i]); return KVMEM_E_INVALID; }
            ids[i] = pg;
        }
    } else {
        int32_t pg = p->free_hint, got = 0;
        for (; pg < p->cfg.max_blocks && got < n_blocks; ++pg)
            if (!p->page_used[pg]) ids[got++] = pg;
        if (got < n_blocks) { set_error("pool has %d free pages, %d needed", got, n_blocks); return KVMEM_E_CAPACITY; }
    }
    return KVMEM_OK;
}

static int append_impl(kvmem_pool_t* p, int32_t session, const void* k, const void* v, int32_t n_blocks,
                       const int32_t* phys_ids, const int32_t* block_pos0, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    if (n_blocks < 0) { set_error("n_blocks is negative"); return KVMEM_E_INVALID; }
    if (n_blocks == 0) return KVMEM_OK;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) { set_error("k and v must be 16-byte aligned device pointers"); return KVMEM_E_INVALID; }
    const int have = p->sess_blocks[session];
    if (!p->sess_reserved[session].empty()) {
        set_error("session %d has %zu reserved blocks in front: commit them (kvmem_commit_blocks) or reset the session", session, p->sess_reserved[session].size());
        return KVMEM_E_STATE;
    }
    if ((int64_t)have + n_blocks > p->cfg.max_blocks_per_session) {
        set_error("session %d holds %d blocks; %d more exceed max_blocks_per_session = %d", session, have, n_blocks,
                  p->cfg.max_blocks_per_session);
        return KVMEM_E_CAPACITY;
    }
    std::vector<int32_t> ids(n_blocks);
    const int rc = choose_pages(p, n_blocks, phys_ids, ids);
    if (rc != KVMEM_OK) return rc;
    if (block_pos0) {
        if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
        for (int i = 0; i < n_blocks; ++i)
            if (block_pos0[i] < 0 || (int64_t)block_pos0[i] + p->cfg.block_tokens > p->cfg.rope_max_positions) {
                set_error("block %d: positions [%d, %d) outside the rotary table [0, %d)", i, block_pos0[i],
                          block_pos0[i] + p->cfg.block_tokens, p->cfg.rope_max_positions);
                return KVMEM_E_INVALID;
            }
    }
    cudaStream_t st = (cudaStream_t)stream;
    int32_t* table = p->tables + (size_t)session * p->cfg.max_blocks_per_session;
    cudaError_t e = cudaMemcpyAsync(table + have, ids.data(), (size_t)n_blocks * 4, cudaMemcpyHostToDevice, st);
    if (e != cudaSuccess) return cuda_fail("block table upload", e);
    const int32_t total = have + n_blocks;
    if (block_pos0) {
        e = cudaMemcpyAsync(p->pos0_dev + (size_t)session * p->cfg.max_blocks_per_session + have, block_pos0,
                            (size_t)n_blocks * 4, cudaMemcpyHostToDevice, st);
        if (e != cudaSuccess) return cuda_fail("block position upload", e);
    }
    e = p->cfg.fp8_pages ? launch_append_fp8(*p, session, have, n_blocks, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, st, block_pos0 != nullptr)
                         : launch_append(*p, session, have, n_blocks, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, st, block_pos0 != nullptr);
    if (e != cudaSuccess) return cuda_fail("append kernel launch", e);
    // the device's block count last: it never covers index rows whose kernel was not enqueued
    e = cudaMemcpyAsync(p->nblocks_dev + session, &total, 4, cudaMemcpyHostToDevice, st);
    if (e != cudaSuccess) return cuda_fail("block count upload", e);
    for (int32_t pg : ids) { p->page_used[pg] = 1; p->sess_pages[session].push_back(pg); }
    if (!phys_ids) p->free_hint = ids.back() + 1;
    p->sess_blocks[session] = total;
    return KVMEM_OK;
}

int kvmem_append_blocks(kvmem_pool_t* p, int32_t session, const void* k, const void* v, int32_t n_blocks,
                        const int32_t* phys_ids, void* stream) {
    return append_impl(p, session, k, v, n_blocks, phys_ids, nullptr, stream);
}

int kvmem_append_blocks_rope(kvmem_pool_t* p, int32_t session, const void* k_roped, const void* v, int32_t n_blocks,
                             const int32_t* phys_ids, const int32_t* block_pos0, void* stream) {
    if (!block_pos0) { set_error("block_pos0 is null"); return KVMEM_E_INVALID; }
    return append_impl(p, session, k_roped, v, n_blocks, phys_ids, block_pos0, stream);
}

int kvmem_rope_rotate(kvmem_pool_t* p, const void* x, void* y, int64_t n_rows, int32_t n_vec, const int32_t* positions,
                      int32_t inverse, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    if (!x || !y || !positions || !aligned(x, 16) || !aligned(y, 16) || n_rows < 0 || n_vec < 1) {
        set_error("kvmem_rope_rotate: null or misaligned pointer, or bad sizes");
        return KVMEM_E_INVALID;
    }
    if (n_rows == 0) return KVMEM_OK;
    cudaError_t e = launch_rope_rotate(*p, (const __nv_bfloat16*)x, (__nv_bfloat16*)y, n_rows, n_vec, positions, inverse,
                                       (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("rotary kernel launch", e);
    return KVMEM_OK;
}

int kvmem_materialize_rope(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids,
                           int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v, int32_t view_cap_tokens,
                           int32_t first_position, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    if (!sel_ids || !n_sel || !view_k || !view_v || !aligned(view_k, 16) || !aligned(view_v, 16)) {
        set_error("kvmem_materialize_rope: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (sel_stride < 1 || view_cap_tokens < p->cfg.block_tokens || view_cap_tokens % p->cfg.block_tokens != 0) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens and sel_stride positive");
        return KVMEM_E_INVALID;
    }
    const int64_t last = (int64_t)first_position + std::min<int64_t>((int64_t)sel_stride * p->cfg.block_tokens, view_cap_tokens);
    if (first_position < 0 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last,
                  p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_gather_rope(*p, session_first, n_sessions, sel_ids, sel_stride, n_sel, (__nv_bfloat16*)view_k,
                                       (__nv_bfloat16*)view_v, view_cap_tokens, first_position, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("rotary gather kernel launch", e);
    return KVMEM_OK;
}

// scoring stage shared by kvmem_score and kvmem_select; *sc_out receives where the scores were written
static int score_impl(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                      float* scores, float score_scale, void* workspace, size_t workspace_bytes, cudaStream_t st, float** sc_out) {
    if (!q || !aligned(q, 16) || !workspace || !aligned(workspace, 256)) {
        set_error("scoring: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1) { set_error("n_q_tokens must be positive"); return KVMEM_E_INVALID; }
    if (p->cfg.head_dim != 128) { set_error("scoring kernels are built for head_dim 128"); return KVMEM_E_UNSUPPORTED; }
    float* sc = nullptr;
    cudaError_t e;
    if (n_q_tokens > kMaxDecodeTokens) {
        // a multi-token chunk makes scoring a dense contraction: tensor-core path
        if (!chunked_scoring_supported(p->cfg, n_q_tokens)) {
            set_error("chunked scoring needs head_dim 128, H/G dividing 128 and n_q_tokens * H/G <= 4096 "
                      "(scores are additive over query tokens: split a longer chunk and add)");
            return KVMEM_E_UNSUPPORTED;
        }
        ChunkWorkspace cw = plan_chunk_workspace(p->cfg, n_sessions, n_q_tokens, (char*)workspace);
        if (workspace_bytes < cw.total) { set_error("select workspace holds %zu bytes, %zu needed", workspace_bytes, cw.total); return KVMEM_E_CAPACITY; }
        sc = scores ? scores : cw.scores;
        e = launch_score_chunked(*p, session_first, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, cw, sc,
                                 p->cfg.max_blocks_per_session, score_scale, st);
    } else {
        ScoreWorkspace ws = plan_score_workspace(p->cfg, n_sessions, n_q_tokens, (char*)workspace);
        if (workspace_bytes < ws.total) { set_error("select workspace holds %zu bytes, %zu needed", workspace_bytes, ws.total); return KVMEM_E_CAPACITY; }
        sc = scores ? scores : ws.scores;
        e = launch_score_decode(*p, session_first, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, ws, sc,
                                p->cfg.max_blocks_per_session, score_scale, st);
    }
    if (e != cudaSuccess) return cuda_fail("score kernel launch", e);
    *sc_out = sc;
    return KVMEM_OK;
}

int kvmem_score(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens, float* scores,
                float score_scale, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!scores) { set_error("scores is null"); return KVMEM_E_INVALID; }
    if (!(score_scale >= 0.0f) || !std::isfinite(score_scale)) { set_error("score_scale must be non-negative and finite (0 selects 1)"); return KVMEM_E_INVALID; }
    float* sc = nullptr;
    return score_impl(p, session_first, n_sessions, q, n_q_tokens, scores, score_scale > 0.0f ? score_scale : 1.0f, workspace,
                      workspace_bytes, (cudaStream_t)stream, &sc);
}

// ---- index in host memory, streamed in tiles

static bool host_score_args_ok(const kvmem_pool_t* p, int32_t n_blocks, int32_t n_q_tokens, int32_t tile_blocks) {
    if (n_blocks < 1 || n_q_tokens < 1 || n_q_tokens > kMaxDecodeTokens) {
        set_error("host-index scoring takes 1..%d query tokens and at least one block", kMaxDecodeTokens);
        return false;
    }
    if (tile_blocks < 128 || tile_blocks % 128 != 0) { set_error("tile_blocks must be a positive multiple of 128"); return false; }
    if (p->cfg.head_dim != 128) { set_error("scoring kernels are built for head_dim 128"); return false; }
    if ((int64_t)p->cfg.n_layers * p->cfg.n_kv_heads * tile_blocks > 0x7fffffffll) { set_error("tile too large"); return false; }
    return true;
}

size_t kvmem_score_host_workspace_bytes(const kvmem_pool_t* p, int32_t n_blocks, int32_t n_q_tokens, int32_t tile_blocks) {
    if (!p || !host_score_args_ok(p, n_blocks, n_q_tokens, tile_blocks)) return 0;
    return plan_host_score(p->cfg, n_blocks, n_q_tokens, tile_blocks, p->sm_count, nullptr).total;
}

size_t kvmem_score_host_staging_bytes(const kvmem_pool_t* p, int32_t tile_blocks) {
    if (!p || !host_score_args_ok(p, 1, 1, tile_blocks)) return 0;
    return plan_host_score(p->cfg, 1, 1, tile_blocks, p->sm_count, nullptr).staging_bytes;
}

int kvmem_score_host_index(kvmem_pool_t* p, const void* index_host, int32_t n_blocks, int32_t index_stride_blocks, const void* q,
                           int32_t n_q_tokens, int32_t tile_blocks, float* scores, void* staging, size_t staging_bytes,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!host_score_args_ok(p, n_blocks, n_q_tokens, tile_blocks)) return KVMEM_E_INVALID;
    if (!index_host || !q || !scores || !staging || !workspace || !aligned(index_host, 16) || !aligned(q, 16) ||
        !aligned(staging, 256) || !aligned(workspace, 256)) {
        set_error("kvmem_score_host_index: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (index_stride_blocks < n_blocks) { set_error("index_stride_blocks is below n_blocks"); return KVMEM_E_INVALID; }
    HostScorePlan plan = plan_host_score(p->cfg, n_blocks, n_q_tokens, tile_blocks, p->sm_count, (char*)workspace);
    if (workspace_bytes < plan.total) { set_error("workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    if (staging_bytes < plan.staging_bytes) { set_error("staging holds %zu bytes, %zu needed", staging_bytes, plan.staging_bytes); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_score_host_index(*p, (const __nv_bfloat16*)index_host, n_blocks, index_stride_blocks,
                                            (const __nv_bfloat16*)q, n_q_tokens, tile_blocks, staging, plan, scores,
                                            (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("host-index scoring", e);
    return KVMEM_OK;
}

int kvmem_topk(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const float* scores, int32_t scores_stride,
               const kvmem_select_params_t* prm, int32_t* sel_ids, int32_t sel_stride, int32_t* n_sel, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!scores || !prm || !sel_ids || !n_sel) { set_error("kvmem_topk: null pointer"); return KVMEM_E_INVALID; }
    if (prm->n_sink_blocks < 0 || prm->n_recent_blocks < 0) { set_error("sink/recent counts must be non-negative"); return KVMEM_E_INVALID; }
    int max_k = 0, max_nb = 0;
    for (int s = session_first; s < session_first + n_sessions; ++s) {
        max_k = std::max(max_k, kvmem_budget_blocks(prm, p->cfg.block_tokens, p->sess_blocks[s]));
        max_nb = std::max(max_nb, p->sess_blocks[s]);
    }
    if (sel_stride < max_k) { set_error("sel_stride %d is below the clamped budget %d", sel_stride, max_k); return KVMEM_E_CAPACITY; }
    if (scores_stride < max_nb) { set_error("scores_stride %d is below the session length %d", scores_stride, max_nb); return KVMEM_E_INVALID; }
    cudaError_t e = launch_topk(*p, session_first, n_sessions, scores, scores_stride, *prm, sel_ids, sel_stride, n_sel,
                                (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("top-k kernel launch", e);
    return KVMEM_OK;
}

int kvmem_select(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                 const kvmem_select_params_t* prm, int32_t* sel_ids, int32_t sel_stride, int32_t* n_sel, float* scores,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!prm || !sel_ids || !n_sel) { set_error("kvmem_select: null pointer"); return KVMEM_E_INVALID; }
    if (prm->n_sink_blocks < 0 || prm->n_recent_blocks < 0) { set_error("sink/recent counts must be non-negative"); return KVMEM_E_INVALID; }
    int max_k = 0;
    for (int s = session_first; s < session_first + n_sessions; ++s)
        max_k = std::max(max_k, kvmem_budget_blocks(prm, p->cfg.block_tokens, p->sess_blocks[s]));
    if (sel_stride < max_k) { set_error("sel_stride %d is below the clamped budget %d", sel_stride, max_k); return KVMEM_E_CAPACITY; }
    cudaStream_t st = (cudaStream_t)stream;
    float* sc = nullptr;
    int rc = score_impl(p, session_first, n_sessions, q, n_q_tokens, scores, 1.0f, workspace, workspace_bytes, st, &sc);
    if (rc != KVMEM_OK) return rc;
    cudaError_t e = launch_topk(*p, session_first, n_sessions, sc, p->cfg.max_blocks_per_session, *prm, sel_ids, sel_stride, n_sel, st);
    if (e != cudaSuccess) return cuda_fail("top-k kernel launch", e);
    return KVMEM_OK;
}

int kvmem_materialize(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids,
                      int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v, int32_t view_cap_tokens,
                      void* stream) {
    if (!pool_live(p) || !pages_are(p, false, "kvmem_materialize")) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!sel_ids || !n_sel || !view_k || !view_v || !aligned(view_k, 16) || !aligned(view_v, 16)) {
        set_error("kvmem_materialize: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (sel_stride < 1 || view_cap_tokens < p->cfg.block_tokens || view_cap_tokens % p->cfg.block_tokens != 0) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens and sel_stride positive");
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_gather(*p, session_first, n_sessions, sel_ids, sel_stride, n_sel, (__nv_bfloat16*)view_k,
                                  (__nv_bfloat16*)view_v, view_cap_tokens, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("gather kernel launch", e);
    return KVMEM_OK;
}

int kvmem_materialize_delta(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* prev_ids, const int32_t* n_prev,
                            const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v,
                            int32_t view_cap_tokens, int32_t* stats, void* stream) {
    if (!pool_live(p) || !pages_are(p, false, "kvmem_materialize_delta")) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!prev_ids || !n_prev || !sel_ids || !n_sel || !view_k || !view_v || !aligned(view_k, 16) || !aligned(view_v, 16)) {
        set_error("kvmem_materialize_delta: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (sel_stride < 1 || view_cap_tokens < p->cfg.block_tokens || view_cap_tokens % p->cfg.block_tokens != 0) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens and sel_stride positive");
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_gather(*p, session_first, n_sessions, sel_ids, sel_stride, n_sel, (__nv_bfloat16*)view_k,
                                  (__nv_bfloat16*)view_v, view_cap_tokens, (cudaStream_t)stream, prev_ids, n_prev, stats);
    if (e != cudaSuccess) return cuda_fail("incremental gather kernel launch", e);
    return KVMEM_OK;
}

int kvmem_view_attend(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const void* view_k,
                      const void* view_v, int32_t view_cap_tokens, const int32_t* n_sel, float scale, float* out,
                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (n_sessions < 1) { set_error("n_sessions must be positive"); return KVMEM_E_INVALID; }
    if (!q || !view_k || !view_v || !n_sel || !out || !lse || !workspace || !aligned(q, 16) || !aligned(view_k, 128) ||
        !aligned(view_v, 128) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_view_attend: null or misaligned pointer (views need 128-byte alignment)");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1) { set_error("n_q_tokens must be positive"); return KVMEM_E_INVALID; }
    if (p->cfg.head_dim != 128) {       // any block size the pool accepts (a multiple of 16): the view is walked in 64-token tiles
        set_error("attention kernel is built for head_dim 128");
        return KVMEM_E_UNSUPPORTED;
    }
    if (n_q_tokens * p->geo.r > 64) { set_error("n_q_tokens * (H/G) = %d exceeds 64 rows per call", n_q_tokens * p->geo.r); return KVMEM_E_UNSUPPORTED; }
    if (view_cap_tokens < p->cfg.block_tokens || view_cap_tokens % p->cfg.block_tokens != 0) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens");
        return KVMEM_E_INVALID;
    }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_attend(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, (const __nv_bfloat16*)view_k,
                                  (const __nv_bfloat16*)view_v, view_cap_tokens, n_sel, scale, out, lse, workspace,
                                  (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("attend kernel launch", e);
    return KVMEM_OK;
}

static void step_staging(const kvmem_pool_config_t& c, int ns, int M, size_t* q_b, size_t* out_b, size_t* lse_b) {
    const size_t rows = (size_t)ns * M * c.n_layers * c.n_q_heads;
    *q_b = align_up(rows * c.head_dim * 2, 256);
    *out_b = align_up(rows * c.head_dim * 4, 256);
    *lse_b = align_up(rows * 4, 256);
}

size_t kvmem_step_staging_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why) || n_sessions < 1 || n_q_tokens < 1) {
        set_error("invalid arguments to kvmem_step_staging_bytes");
        return 0;
    }
    size_t a, b, c;
    step_staging(*cfg, n_sessions, n_q_tokens, &a, &b, &c);
    return a + b + c;
}

// the device-side address of a host buffer that the GPU can write directly (pinned and mapped), else null
static float* mapped_host_pointer(float* host) {
    cudaPointerAttributes at{};
    if (cudaPointerGetAttributes(&at, host) != cudaSuccess) { (void)cudaGetLastError(); return nullptr; }
    if (at.type != cudaMemoryTypeHost || !at.devicePointer) return nullptr;
    return static_cast<float*>(at.devicePointer);
}

int kvmem_recall_step_host(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q_host,
                           int32_t n_q_tokens, const kvmem_select_params_t* prm, int32_t* sel_ids, int32_t sel_stride,
                           int32_t* n_sel, void* view_k, void* view_v, int32_t view_cap_tokens, float scale,
                           float* out_host, float* lse_host, void* staging, size_t staging_bytes, void* select_ws,
                           size_t select_ws_bytes, void* attend_ws, size_t attend_ws_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!q_host || !out_host || !lse_host || !staging || !aligned(staging, 256) || n_q_tokens < 1) {
        set_error("kvmem_recall_step_host: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    size_t q_b, out_b, lse_b;
    step_staging(p->cfg, n_sessions, n_q_tokens, &q_b, &out_b, &lse_b);
    if (staging_bytes < q_b + out_b + lse_b) { set_error("staging holds %zu bytes, %zu needed", staging_bytes, q_b + out_b + lse_b); return KVMEM_E_CAPACITY; }
    char* sb = (char*)staging;
    void* q_dev = sb;
    float* out_dev = (float*)(sb + q_b);
    float* lse_dev = (float*)(sb + q_b + out_b);
    const size_t rows = (size_t)n_sessions * n_q_tokens * p->cfg.n_layers * p->cfg.n_q_heads;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaMemcpyAsync(q_dev, q_host, rows * p->cfg.head_dim * 2, cudaMemcpyHostToDevice, st);
    if (e != cudaSuccess) return cuda_fail("query upload", e);
    int rc = kvmem_select(p, session_first, n_sessions, q_dev, n_q_tokens, prm, sel_ids, sel_stride, n_sel, nullptr,
                          select_ws, select_ws_bytes, stream);
    if (rc != KVMEM_OK) return rc;
    // Result buffers in pinned, device-mapped host memory are written by the merge kernel itself (the stores cross
    // PCIe as they are issued and are complete when the stream is): two copy operations less on the critical path
    // of a synchronous step.  Anything else (pageable memory) takes the staged copies.
    float* out_map = mapped_host_pointer(out_host);
    float* lse_map = mapped_host_pointer(lse_host);
    const bool direct = out_map && lse_map && aligned(out_map, 16);
    rc = kvmem_materialize_attend(p, session_first, n_sessions, q_dev, n_q_tokens, sel_ids, sel_stride, n_sel, view_k, view_v,
                                  view_cap_tokens, scale, direct ? out_map : out_dev, direct ? lse_map : lse_dev, attend_ws,
                                  attend_ws_bytes, stream);
    if (rc != KVMEM_OK) return rc;
    if (!direct) {
        e = cudaMemcpyAsync(out_host, out_dev, rows * p->cfg.head_dim * 4, cudaMemcpyDeviceToHost, st);
        if (e == cudaSuccess) e = cudaMemcpyAsync(lse_host, lse_dev, rows * 4, cudaMemcpyDeviceToHost, st);
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return cuda_fail("result download", e);
    return KVMEM_OK;
}

int kvmem_set_option(const char* name, int32_t value) {
    if (!name) { set_error("option name is null"); return KVMEM_E_INVALID; }
    if (strcmp(name, "gather_mode") == 0 && (value == 0 || value == 1)) { g_gather_mode = value; return KVMEM_OK; }
    if (strcmp(name, "chunk_poly") == 0 && (value == 0 || (value >= 2 && value <= 5))) { g_chunk_poly = value; return KVMEM_OK; }
    if (strcmp(name, "topk_cluster") == 0 && (value == 0 || value == 1)) { g_topk_cluster = value; return KVMEM_OK; }
    if (strcmp(name, "topk_items") == 0 && (value == 0 || value == 1 || value == 2 || value == 4 || value == 8 || value == 16)) {
        g_topk_items = value;
        return KVMEM_OK;
    }
    if (strcmp(name, "gather_ctas") == 0 && value >= 0) { g_gather_ctas = value; return KVMEM_OK; }
    if (strcmp(name, "attend_lookahead") == 0 && value >= 0 && value <= 8) { g_attend_lookahead = value; return KVMEM_OK; }
    if (strcmp(name, "attend_landed") == 0 && (value >= -1 && value <= 1)) { g_attend_landed = value; return KVMEM_OK; }
    if (strcmp(name, "attend_splits") == 0 && value >= 0 && value <= 64) { g_attend_splits = value; return KVMEM_OK; }
    if (strcmp(name, "pdl") == 0 && (value == 0 || value == 1)) { g_pdl = value; return KVMEM_OK; }
    if (strcmp(name, "score_mode") == 0 && (value == 0 || value == 1)) { g_score_mode = value; return KVMEM_OK; }
    set_error("unknown option or value: %s = %d", name, value);
    return KVMEM_E_INVALID;
}

// rope_first_position < 0: plain views; otherwise the position-consistent fused pass (in-block key layout)
static int materialize_attend_impl(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                                   const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v,
                                   int32_t view_cap_tokens, int32_t rope_first_position, float scale, float* out, float* lse,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p) || !pages_are(p, false, "kvmem_materialize_attend")) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!q || !sel_ids || !n_sel || !view_k || !view_v || !out || !lse || !workspace || !aligned(q, 16) ||
        !aligned(view_k, 128) || !aligned(view_v, 128) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_materialize_attend: null or misaligned pointer (views need 128-byte alignment)");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1 || sel_stride < 1) { set_error("n_q_tokens and sel_stride must be positive"); return KVMEM_E_INVALID; }
    if (!paged_block_size_ok(p, rope_first_position >= 0 && p->cfg.rope_in_block_keys, "kvmem_materialize_attend")) return KVMEM_E_UNSUPPORTED;
    if (n_q_tokens * p->geo.r > (rope_first_position >= 0 ? 16 : 64)) { set_error("n_q_tokens * (H/G) = %d exceeds %d rows per call", n_q_tokens * p->geo.r, rope_first_position >= 0 ? 16 : 64); return KVMEM_E_UNSUPPORTED; }
    if (view_cap_tokens < p->cfg.block_tokens || view_cap_tokens % p->cfg.block_tokens != 0) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens");
        return KVMEM_E_INVALID;
    }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if ((int64_t)p->cfg.max_blocks * 2 * p->cfg.n_layers * p->cfg.n_kv_heads * p->cfg.block_tokens > 0x7fffffffll) {
        set_error("page pool too large for 32-bit TMA row coordinates");
        return KVMEM_E_UNSUPPORTED;
    }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_attend(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, (const __nv_bfloat16*)view_k,
                                  (const __nv_bfloat16*)view_v, view_cap_tokens, n_sel, scale, out, lse, workspace,
                                  (cudaStream_t)stream, sel_ids, sel_stride, session_first, nullptr, rope_first_position);
    if (e != cudaSuccess) return cuda_fail("fused materialize+attend kernel launch", e);
    return KVMEM_OK;
}

int kvmem_materialize_attend(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                             const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v,
                             int32_t view_cap_tokens, float scale, float* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
    return materialize_attend_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, view_k, view_v,
                                   view_cap_tokens, -1, scale, out, lse, workspace, workspace_bytes, stream);
}

int kvmem_materialize_attend_rope(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                                  const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, void* view_k, void* view_v,
                                  int32_t view_cap_tokens, int32_t first_position, float scale, float* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    if (sel_stride < 1 || view_cap_tokens < 1) { set_error("sel_stride and view_cap_tokens must be positive"); return KVMEM_E_INVALID; }
    const int64_t last = (int64_t)first_position + std::min<int64_t>((int64_t)sel_stride * p->cfg.block_tokens, view_cap_tokens);
    if (first_position < 0 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last,
                  p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    // One pass either way: on the in-block layout every K tile is rotated by its block position on its way through shared
    // memory; raw keys are rotated by the consumer warps on their way to the tensor cores and handed back for the store.
    // The pass walks whole 64-token tiles and fetches rotary rows up to the 49th position of the last one (the bound is
    // kept at the whole tile).
    if (!p->cfg.rope_in_block_keys) {
        const int64_t tiles_end = (int64_t)first_position + (std::min<int64_t>((int64_t)sel_stride * p->cfg.block_tokens, view_cap_tokens) + 63) / 64 * 64;
        if (tiles_end > p->cfg.rope_max_positions) {
            set_error("the last 64-token tile of the view reaches position %lld, outside the rotary table [0, %d)", (long long)tiles_end,
                      p->cfg.rope_max_positions);
            return KVMEM_E_INVALID;
        }
    }
    return materialize_attend_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, view_k, view_v,
                                   view_cap_tokens, first_position, scale, out, lse, workspace, workspace_bytes, stream);
}

static int paged_attend_impl(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                             const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, int32_t rope_first_position,
                             float scale, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p) || !pages_are(p, false, "kvmem_paged_attend")) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!q || !sel_ids || !n_sel || !out || !lse || !workspace || !aligned(q, 16) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_paged_attend: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1 || sel_stride < 1) { set_error("n_q_tokens and sel_stride must be positive"); return KVMEM_E_INVALID; }
    if (!paged_block_size_ok(p, false, "kvmem_paged_attend")) return KVMEM_E_UNSUPPORTED;     // the query-rotating mode handles every block size too
    if (n_q_tokens * p->geo.r > (rope_first_position >= 0 ? 16 : 64)) { set_error("n_q_tokens * (H/G) = %d exceeds %d rows per call", n_q_tokens * p->geo.r, rope_first_position >= 0 ? 16 : 64); return KVMEM_E_UNSUPPORTED; }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if ((int64_t)p->cfg.max_blocks * 2 * p->cfg.n_layers * p->cfg.n_kv_heads * p->cfg.block_tokens > 0x7fffffffll) {
        set_error("page pool too large for 32-bit TMA row coordinates");
        return KVMEM_E_UNSUPPORTED;
    }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    // the "view" is only virtual here: its length bound is sel_stride blocks
    const int64_t cap_tokens = (int64_t)sel_stride * p->cfg.block_tokens;
    if (cap_tokens > 0x7fffffffll) { set_error("sel_stride too large"); return KVMEM_E_INVALID; }
    cudaError_t e = launch_attend(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, nullptr, nullptr, (int)cap_tokens, n_sel,
                                  scale, out, lse, workspace, (cudaStream_t)stream, sel_ids, sel_stride, session_first, nullptr,
                                  rope_first_position);
    if (e != cudaSuccess) return cuda_fail("paged attention kernel launch", e);
    return KVMEM_OK;
}

int kvmem_paged_attend(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                       const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, float scale, float* out, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
    return paged_attend_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, -1, scale, out, lse,
                             workspace, workspace_bytes, stream);
}

int kvmem_paged_attend_rope(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                            const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, int32_t first_position,
                            float scale, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    // the pass walks whole 64-token tiles: the last tile fetches rotary rows up to its 49th position (bound kept at the whole tile)
    const int64_t last = (int64_t)first_position + ((int64_t)sel_stride * p->cfg.block_tokens + 63) / 64 * 64;
    if (first_position < 0 || sel_stride < 1 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last,
                  p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    return paged_attend_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, first_position, scale, out,
                             lse, workspace, workspace_bytes, stream);
}

int kvmem_working_set_delta(kvmem_pool_t* p, int32_t n_sessions, const int32_t* prev_ids, const int32_t* n_prev,
                            const int32_t* next_ids, const int32_t* n_next, int32_t stride, int32_t* retained,
                            int32_t* incoming, int32_t* outgoing, int32_t* counts, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (n_sessions < 1 || stride < 1 || !prev_ids || !n_prev || !next_ids || !n_next || !retained || !incoming || !outgoing ||
        !counts) {
        set_error("kvmem_working_set_delta: null pointer or non-positive size");
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_working_set_delta(*p, n_sessions, prev_ids, n_prev, next_ids, n_next, stride, retained, incoming,
                                             outgoing, counts, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("working-set delta kernel launch", e);
    return KVMEM_OK;
}

// ---- FP8 execution view ----

static int fp8_common_ok(kvmem_pool_t* p, int32_t view_cap_tokens, float k_scale, float v_scale, const char* who) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.head_dim != 128 || p->cfg.block_tokens != 64) {
        set_error("%s: the FP8 view kernels are built for head_dim 128 and 64-token blocks", who);
        return KVMEM_E_UNSUPPORTED;
    }
    if (view_cap_tokens < 64 || view_cap_tokens % 64 != 0) { set_error("%s: view_cap_tokens must be a positive multiple of 64", who); return KVMEM_E_INVALID; }
    if (!(k_scale > 0.0f) || !(v_scale > 0.0f) || !std::isfinite(k_scale) || !std::isfinite(v_scale)) {
        set_error("%s: scales must be positive and finite", who);
        return KVMEM_E_INVALID;
    }
    return KVMEM_OK;
}

int kvmem_materialize_fp8(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids, int32_t sel_stride,
                          const int32_t* n_sel, void* view_k8, void* view_v8t, int32_t view_cap_tokens, float k_scale,
                          float v_scale, void* stream) {
    const int rc = fp8_common_ok(p, view_cap_tokens, k_scale, v_scale, "kvmem_materialize_fp8");
    if (rc != KVMEM_OK) return rc;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!sel_ids || !n_sel || !view_k8 || !view_v8t || !aligned(view_k8, 128) || !aligned(view_v8t, 128) || sel_stride < 1) {
        set_error("kvmem_materialize_fp8: null or misaligned pointer (views need 128-byte alignment), or sel_stride < 1");
        return KVMEM_E_INVALID;
    }
    if (p->cfg.fp8_pages && (k_scale != p->cfg.fp8_k_scale || v_scale != p->cfg.fp8_v_scale)) {
        set_error("kvmem_materialize_fp8: the pool's pages were quantised with scales %g / %g, not %g / %g", p->cfg.fp8_k_scale,
                  p->cfg.fp8_v_scale, k_scale, v_scale);
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_gather_fp8(*p, session_first, n_sessions, sel_ids, sel_stride, n_sel, (uint8_t*)view_k8,
                                      (uint8_t*)view_v8t, view_cap_tokens, k_scale, v_scale, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("FP8 gather kernel launch", e);
    return KVMEM_OK;
}

int kvmem_materialize_fp8_rope(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* sel_ids, int32_t sel_stride,
                               const int32_t* n_sel, void* view_k8, void* view_v8t, int32_t view_cap_tokens, int32_t first_position,
                               float k_scale, float v_scale, void* stream) {
    const int rc = fp8_common_ok(p, view_cap_tokens, k_scale, v_scale, "kvmem_materialize_fp8_rope");
    if (rc != KVMEM_OK) return rc;
    if (!pages_are(p, false, "kvmem_materialize_fp8_rope")) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!sel_ids || !n_sel || !view_k8 || !view_v8t || !aligned(view_k8, 128) || !aligned(view_v8t, 128) || sel_stride < 1) {
        set_error("kvmem_materialize_fp8_rope: null or misaligned pointer (views need 128-byte alignment), or sel_stride < 1");
        return KVMEM_E_INVALID;
    }
    const int64_t last = (int64_t)first_position + std::min<int64_t>((int64_t)sel_stride * 64, view_cap_tokens);
    if (first_position < 0 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last, p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    cudaError_t e = launch_gather_fp8(*p, session_first, n_sessions, sel_ids, sel_stride, n_sel, (uint8_t*)view_k8,
                                      (uint8_t*)view_v8t, view_cap_tokens, k_scale, v_scale, (cudaStream_t)stream, first_position);
    if (e != cudaSuccess) return cuda_fail("rotating FP8 gather kernel launch", e);
    return KVMEM_OK;
}

int kvmem_view_attend_fp8(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const void* view_k8,
                          const void* view_v8t, int32_t view_cap_tokens, const int32_t* n_sel, float scale, float k_scale,
                          float v_scale, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = fp8_common_ok(p, view_cap_tokens, k_scale, v_scale, "kvmem_view_attend_fp8");
    if (rc != KVMEM_OK) return rc;
    if (n_sessions < 1 || n_q_tokens < 1) { set_error("n_sessions and n_q_tokens must be positive"); return KVMEM_E_INVALID; }
    if (!q || !view_k8 || !view_v8t || !n_sel || !out || !lse || !workspace || !aligned(q, 16) || !aligned(view_k8, 128) ||
        !aligned(view_v8t, 128) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_view_attend_fp8: null or misaligned pointer (views need 128-byte alignment)");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens * p->geo.r > 16) { set_error("n_q_tokens * (H/G) = %d exceeds 16 rows per call", n_q_tokens * p->geo.r); return KVMEM_E_UNSUPPORTED; }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if ((int64_t)n_sessions * p->cfg.n_layers * p->cfg.n_kv_heads * view_cap_tokens > 0x7fffffffll) {
        set_error("view too large for 32-bit TMA row coordinates");
        return KVMEM_E_UNSUPPORTED;
    }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_attend_fp8(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, (const uint8_t*)view_k8,
                                      (const uint8_t*)view_v8t, view_cap_tokens, n_sel, scale, k_scale, v_scale, out, lse,
                                      workspace, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("FP8 attention kernel launch", e);
    return KVMEM_OK;
}

static int paged_attend_fp8_impl(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                                 const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, int32_t rope_first_position,
                                 float scale, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p) || !pages_are(p, true, "kvmem_paged_attend_fp8")) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!q || !sel_ids || !n_sel || !out || !lse || !workspace || !aligned(q, 16) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_paged_attend_fp8: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1 || sel_stride < 1) { set_error("n_q_tokens and sel_stride must be positive"); return KVMEM_E_INVALID; }
    if (n_q_tokens * p->geo.r > 16) { set_error("n_q_tokens * (H/G) = %d exceeds 16 rows per call", n_q_tokens * p->geo.r); return KVMEM_E_UNSUPPORTED; }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if ((int64_t)p->cfg.max_blocks * 2 * p->cfg.n_layers * p->cfg.n_kv_heads * 64 > 0x7fffffffll) {
        set_error("page pool too large for 32-bit TMA row coordinates");
        return KVMEM_E_UNSUPPORTED;
    }
    if ((int64_t)sel_stride * 64 > 0x7fffffffll) { set_error("sel_stride too large"); return KVMEM_E_INVALID; }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_attend_fp8(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, nullptr, nullptr, sel_stride * 64, n_sel,
                                      scale, p->cfg.fp8_k_scale, p->cfg.fp8_v_scale, out, lse, workspace, (cudaStream_t)stream,
                                      sel_ids, sel_stride, session_first, rope_first_position);
    if (e != cudaSuccess) return cuda_fail("paged FP8 attention kernel launch", e);
    return KVMEM_OK;
}

int kvmem_paged_attend_fp8(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                           const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, float scale, float* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* stream) {
    return paged_attend_fp8_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, -1, scale, out, lse,
                                 workspace, workspace_bytes, stream);
}

int kvmem_paged_attend_fp8_rope(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                                const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, int32_t first_position,
                                float scale, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!p->cfg.fp8_pages || !p->cfg.rope_in_block_keys) {
        set_error("kvmem_paged_attend_fp8_rope needs a pool with fp8_pages and rope_in_block_keys");
        return KVMEM_E_STATE;
    }
    const int64_t last = (int64_t)first_position + (int64_t)sel_stride * p->cfg.block_tokens;
    if (first_position < 0 || sel_stride < 1 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last,
                  p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    return paged_attend_fp8_impl(p, session_first, n_sessions, q, n_q_tokens, sel_ids, sel_stride, n_sel, first_position, scale,
                                 out, lse, workspace, workspace_bytes, stream);
}

int kvmem_materialize_attend_fp8(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                                 const int32_t* sel_ids, int32_t sel_stride, const int32_t* n_sel, void* view_k8, void* view_v8t,
                                 int32_t view_cap_tokens, float scale, float* out, float* lse, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.head_dim != 128 || p->cfg.block_tokens != 64) {
        set_error("kvmem_materialize_attend_fp8: the FP8 view kernels are built for head_dim 128 and 64-token blocks");
        return KVMEM_E_UNSUPPORTED;
    }
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    // a bf16 repository is quantised on the way with the pool's scales, 1 where the configuration leaves them unset
    const float k_scale = p->cfg.fp8_k_scale > 0.0f && std::isfinite(p->cfg.fp8_k_scale) ? p->cfg.fp8_k_scale : 1.0f;
    const float v_scale = p->cfg.fp8_v_scale > 0.0f && std::isfinite(p->cfg.fp8_v_scale) ? p->cfg.fp8_v_scale : 1.0f;
    if (!q || !sel_ids || !n_sel || !view_k8 || !view_v8t || !out || !lse || !workspace || !aligned(q, 16) || !aligned(view_k8, 128) ||
        !aligned(view_v8t, 128) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_materialize_attend_fp8: null or misaligned pointer (views need 128-byte alignment)");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1 || sel_stride < 1) { set_error("n_q_tokens and sel_stride must be positive"); return KVMEM_E_INVALID; }
    if (view_cap_tokens < 64 || view_cap_tokens % 64 != 0) { set_error("view_cap_tokens must be a positive multiple of 64"); return KVMEM_E_INVALID; }
    if (n_q_tokens * p->geo.r > 16) { set_error("n_q_tokens * (H/G) = %d exceeds 16 rows per call", n_q_tokens * p->geo.r); return KVMEM_E_UNSUPPORTED; }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if ((int64_t)p->cfg.max_blocks * 2 * p->cfg.n_layers * p->cfg.n_kv_heads * 64 > 0x7fffffffll ||
        (int64_t)n_sessions * p->cfg.n_layers * p->cfg.n_kv_heads * view_cap_tokens > 0x7fffffffll) {
        set_error("page pool or view too large for 32-bit TMA row coordinates");
        return KVMEM_E_UNSUPPORTED;
    }
    AttendPlan plan = plan_attend(p->cfg, n_sessions, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    cudaError_t e = launch_attend_fp8(*p, n_sessions, (const __nv_bfloat16*)q, n_q_tokens, (const uint8_t*)view_k8,
                                      (const uint8_t*)view_v8t, view_cap_tokens, n_sel, scale, k_scale, v_scale,
                                      out, lse, workspace, (cudaStream_t)stream, sel_ids, sel_stride, session_first);
    if (e != cudaSuccess) return cuda_fail("fused FP8 materialize+attend kernel launch", e);
    return KVMEM_OK;
}

// ---- execution cache: working-set reuse with bounded delta re-RoPE ----

static int cache_ok(kvmem_pool_t* p, const void* cache, size_t cache_bytes, int32_t cap_blocks, const char* who) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("%s: the pool was created without rotary support", who); return KVMEM_E_STATE; }
    if (cap_blocks < 1 || cap_blocks > 32768) { set_error("%s: cap_blocks must be in [1, 32768]", who); return KVMEM_E_INVALID; }
    if (!cache || !aligned(cache, 256)) { set_error("%s: cache is null or not 256-byte aligned", who); return KVMEM_E_INVALID; }
    const size_t need = cache_layout(p->lay.page_elems, cap_blocks).total;
    if (cache_bytes < need) { set_error("%s: cache holds %zu bytes, %zu needed", who, cache_bytes, need); return KVMEM_E_CAPACITY; }
    return KVMEM_OK;
}

size_t kvmem_view_cache_bytes(const kvmem_pool_t* p, int32_t cap_blocks) {
    if (!p || cap_blocks < 1 || cap_blocks > 32768) return 0;
    return cache_layout(p->lay.page_elems, cap_blocks).total;
}

int kvmem_view_cache_layout(const kvmem_pool_t* p, int32_t cap_blocks, size_t* offsets) {
    if (!p || !offsets || cap_blocks < 1 || cap_blocks > 32768) { set_error("kvmem_view_cache_layout: bad argument"); return KVMEM_E_INVALID; }
    const CacheLayout c = cache_layout(p->lay.page_elems, cap_blocks);
    offsets[0] = c.pages; offsets[1] = c.slot_block; offsets[2] = c.slot_pos; offsets[3] = c.slot_cnt;
    offsets[4] = c.view_slots; offsets[5] = c.n_view;
    return KVMEM_OK;
}

int kvmem_view_cache_reset(kvmem_pool_t* p, void* cache, size_t cache_bytes, int32_t cap_blocks, void* stream) {
    const int rc = cache_ok(p, cache, cache_bytes, cap_blocks, "kvmem_view_cache_reset");
    if (rc != KVMEM_OK) return rc;
    cudaError_t e = launch_view_cache_reset(*p, cache, cap_blocks, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("execution-cache reset kernel launch", e);
    return KVMEM_OK;
}

int kvmem_view_cache_update(kvmem_pool_t* p, int32_t session, const int32_t* sel_ids, const int32_t* n_sel, void* cache,
                            size_t cache_bytes, int32_t cap_blocks, int32_t max_delta_ropes, int32_t first_position,
                            int32_t* stats, void* stream) {
    const int rc = cache_ok(p, cache, cache_bytes, cap_blocks, "kvmem_view_cache_update");
    if (rc != KVMEM_OK) return rc;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    if (!sel_ids || !n_sel) { set_error("kvmem_view_cache_update: null pointer"); return KVMEM_E_INVALID; }
    if (max_delta_ropes < 0) { set_error("max_delta_ropes must be non-negative"); return KVMEM_E_INVALID; }
    const int64_t last = (int64_t)first_position + (int64_t)cap_blocks * p->cfg.block_tokens;
    if (first_position < 0 || last > p->cfg.rope_max_positions) {
        set_error("compact positions [%d, %lld) outside the rotary table [0, %d)", first_position, (long long)last,
                  p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    if (p->cfg.head_dim % 16 != 0) { set_error("rotary kernels need head_dim to be a multiple of 16"); return KVMEM_E_UNSUPPORTED; }
    cudaError_t e = launch_view_cache_update(*p, session, sel_ids, n_sel, cache, cap_blocks, max_delta_ropes, first_position,
                                             stats, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("execution-cache update kernel launch", e);
    return KVMEM_OK;
}

int kvmem_view_cache_attend(kvmem_pool_t* p, const void* q, int32_t n_q_tokens, void* cache, size_t cache_bytes,
                            int32_t cap_blocks, float scale, float* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
    const int rc = cache_ok(p, cache, cache_bytes, cap_blocks, "kvmem_view_cache_attend");
    if (rc != KVMEM_OK) return rc;
    if (!q || !out || !lse || !workspace || !aligned(q, 16) || !aligned(workspace, 256) || !aligned(out, 16)) {
        set_error("kvmem_view_cache_attend: null or misaligned pointer");
        return KVMEM_E_INVALID;
    }
    if (n_q_tokens < 1) { set_error("n_q_tokens must be positive"); return KVMEM_E_INVALID; }
    if (!paged_block_size_ok(p, false, "kvmem_view_cache_attend")) return KVMEM_E_UNSUPPORTED;
    if (n_q_tokens * p->geo.r > 64) { set_error("n_q_tokens * (H/G) = %d exceeds 64 rows per call", n_q_tokens * p->geo.r); return KVMEM_E_UNSUPPORTED; }
    if (!(scale >= 0.0f)) { set_error("scale must be non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    AttendPlan plan = plan_attend(p->cfg, 1, n_q_tokens, p->sm_count);
    if (workspace_bytes < plan.total) { set_error("attend workspace holds %zu bytes, %zu needed", workspace_bytes, plan.total); return KVMEM_E_CAPACITY; }
    PagedSource src{};
    view_cache_paged_source(*p, cache, cap_blocks, &src);
    const int64_t cap_tokens = (int64_t)cap_blocks * p->cfg.block_tokens;
    cudaError_t e = launch_attend(*p, 1, (const __nv_bfloat16*)q, n_q_tokens, nullptr, nullptr, (int)cap_tokens, src.n_sel, scale,
                                  out, lse, workspace, (cudaStream_t)stream, src.sel_ids, cap_blocks, 0, &src);
    if (e != cudaSuccess) return cuda_fail("execution-cache attention kernel launch", e);
    return KVMEM_OK;
}

// ---- decode over a view: drafted tokens, accumulated weights, eviction ----

// [p, p + n) and [q, q + m) share a byte
static bool overlap(const void* p, size_t n, const void* q, size_t m) {
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + m && b < a + n;
}

// What the attention calls refuse for its size alone, and their workspace sizes with them.  weights: the call that accumulates
// them; view_cap_tokens 0: a view of any length.  KVMEM_OK, or the status with its message set.
static int tree_sizes(const kvmem_pool_config_t& c, int32_t n_sessions, int32_t n_q_tokens, bool weights, int32_t view_cap_tokens) {
    if (n_sessions < 1 || n_sessions > 65535) { set_error("n_sessions must be in [1, 65535]"); return KVMEM_E_INVALID; }
    if (n_q_tokens < 1 || n_q_tokens > kMaxDrafted) { set_error("n_q_tokens must be in [1, %d]", kMaxDrafted); return KVMEM_E_INVALID; }
    if (view_cap_tokens && (view_cap_tokens < c.block_tokens || view_cap_tokens % c.block_tokens != 0)) {
        set_error("view_cap_tokens must be a positive multiple of block_tokens");
        return KVMEM_E_INVALID;
    }
    if (c.head_dim != 128) { set_error("the attention kernel is built for head_dim 128"); return KVMEM_E_UNSUPPORTED; }
    const long long rows = (long long)n_q_tokens * (c.n_q_heads / c.n_kv_heads), most = weights ? 64 : 65536;
    if (rows > most) { set_error("n_q_tokens * (H/G) = %lld exceeds %lld rows per KV head", rows, most); return KVMEM_E_UNSUPPORTED; }
    if (weights && view_cap_tokens > (1 << 23)) { set_error("views of more than 2^23 tokens are not supported"); return KVMEM_E_UNSUPPORTED; }
    return KVMEM_OK;
}

static int line_fits(const kvmem_pool_config_t& c, int32_t n_sessions, int32_t n_q_tokens, int32_t cap_tokens, int32_t tail_cap_tokens) {
    if (tree_line_fits(c, n_sessions, n_q_tokens, cap_tokens, tail_cap_tokens)) return KVMEM_OK;
    set_error("%d sessions of up to %d + %d tokens are more than 2^30 units of a line of tiles", n_sessions, cap_tokens, tail_cap_tokens);
    return KVMEM_E_UNSUPPORTED;
}

static size_t tree_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens, int32_t mass_cap, const char* who) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why)) { set_error("invalid arguments to %s", who); return 0; }
    if (tree_sizes(*cfg, n_sessions, n_q_tokens, mass_cap > 0, mass_cap) != KVMEM_OK ||
        line_fits(*cfg, n_sessions, n_q_tokens, mass_cap ? mass_cap : cfg->block_tokens, 0) != KVMEM_OK) return 0;
    return tree_workspace_bytes(*cfg, n_sessions, n_q_tokens, mass_cap);
}

size_t kvmem_tree_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens) {
    return tree_bytes(cfg, n_sessions, n_q_tokens, 0, "kvmem_tree_workspace_bytes");
}

size_t kvmem_mass_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens, int32_t view_cap_tokens) {
    if (view_cap_tokens < 1) { set_error("view_cap_tokens must be positive"); return 0; }
    return tree_bytes(cfg, n_sessions, n_q_tokens, view_cap_tokens, "kvmem_mass_workspace_bytes");
}

// what the three attention calls check alike; fills the arguments that do not depend on where the keys live
static int tree_common(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const int32_t* n_q,
                       const uint64_t* mask, const int32_t* n_sel, const kvmem_tail_t* tail, float scale, void* out, float* lse,
                       const char* who, TreeArgs* a) {
    if (!q || !n_sel || !out || !lse || !aligned(q, 16) || !aligned(out, 16)) {
        set_error("%s: null or misaligned pointer", who);
        return KVMEM_E_INVALID;
    }
    if (!(scale >= 0.0f) || !std::isfinite(scale)) { set_error("scale must be finite and non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    if (tail) {
        if (!tail->k || !tail->v || !tail->n_tokens || !aligned(tail->k, 16) || !aligned(tail->v, 16)) {
            set_error("%s: null or misaligned tail pointer", who);
            return KVMEM_E_INVALID;
        }
        if (tail->cap_tokens < n_q_tokens || (int64_t)tail->cap_tokens * n_sessions > INT32_MAX) {
            set_error("the tail holds %d tokens per session: at least n_q_tokens = %d are needed, and n_sessions * cap_tokens must stay below 2^31",
                      tail->cap_tokens, n_q_tokens);
            return KVMEM_E_INVALID;
        }
    } else if (mask) {
        set_error("a mask says which drafted keys a token sees: it needs a tail that holds them");
        return KVMEM_E_INVALID;
    }
    const Geometry& g = p->geo;
    a->q = (const __nv_bfloat16*)q; a->n_q = n_q; a->mask = (const unsigned long long*)mask; a->n_sel = n_sel;
    if (tail) { a->tail_k = (const __nv_bfloat16*)tail->k; a->tail_v = (const __nv_bfloat16*)tail->v; a->n_tail = tail->n_tokens; a->tail_cap = tail->cap_tokens; }
    a->out = (__nv_bfloat16*)out; a->lse = lse; a->status = p->status_dev;
    a->ns = n_sessions; a->M = n_q_tokens; a->L = g.L; a->H = g.H; a->G = g.G; a->r = g.r; a->rows = n_q_tokens * g.r; a->B = g.B;
    a->scale = scale > 0.0f ? scale : 1.0f / sqrtf((float)g.d);
    return KVMEM_OK;
}

static int tree_view(const void* view_k, const void* view_v, int32_t view_cap_tokens, const char* who, TreeArgs* a) {
    if (!view_k || !view_v || !aligned(view_k, 128) || !aligned(view_v, 128)) {
        set_error("%s: null or misaligned pointer (views need 128-byte alignment)", who);
        return KVMEM_E_INVALID;
    }
    a->view_k = (const __nv_bfloat16*)view_k; a->view_v = (const __nv_bfloat16*)view_v; a->cap = view_cap_tokens;
    return KVMEM_OK;
}

// limits of the whole call, the workspace, the launches
static int tree_run(kvmem_pool_t* p, const TreeArgs& a, void* workspace, size_t workspace_bytes, void* stream, const char* who) {
    const int rc = line_fits(p->cfg, a.ns, a.M, a.cap, a.tail_cap);
    if (rc != KVMEM_OK) return rc;
    if (!workspace || !aligned(workspace, 256)) { set_error("%s: null or misaligned workspace", who); return KVMEM_E_INVALID; }
    const size_t need = tree_workspace_bytes(p->cfg, a.ns, a.M, a.mass ? a.cap : 0);
    if (workspace_bytes < need) { set_error("%s: the workspace holds %zu bytes, %zu needed", who, workspace_bytes, need); return KVMEM_E_CAPACITY; }
    const cudaError_t e = launch_tree(*p, a, workspace, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(who, e);
    return KVMEM_OK;
}

int kvmem_view_tree_attend(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const int32_t* n_q,
                           const uint64_t* mask, const void* view_k, const void* view_v, int32_t view_cap_tokens,
                           const int32_t* n_sel, const kvmem_tail_t* tail, float scale, void* out, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
    const char* who = "kvmem_view_tree_attend";
    if (!pool_live(p)) return KVMEM_E_STATE;
    TreeArgs a{};
    int rc = tree_sizes(p->cfg, n_sessions, n_q_tokens, false, view_cap_tokens ? view_cap_tokens : -1);
    if (rc == KVMEM_OK) rc = tree_common(p, n_sessions, q, n_q_tokens, n_q, mask, n_sel, tail, scale, out, lse, who, &a);
    if (rc == KVMEM_OK) rc = tree_view(view_k, view_v, view_cap_tokens, who, &a);
    return rc == KVMEM_OK ? tree_run(p, a, workspace, workspace_bytes, stream, who) : rc;
}

int kvmem_paged_tree_attend(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const void* q, int32_t n_q_tokens,
                            const int32_t* n_q, const uint64_t* mask, const int32_t* sel_ids, int32_t sel_stride,
                            const int32_t* n_sel, const kvmem_tail_t* tail, float scale, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!pages_are(p, false, "kvmem_paged_tree_attend")) return KVMEM_E_STATE;
    if (p->cfg.rope_in_block_keys) {
        set_error("kvmem_paged_tree_attend has no positions for keys rotated by their offset in the block: kvmem_materialize_rope and kvmem_view_tree_attend");
        return KVMEM_E_STATE;
    }
    const char* who = "kvmem_paged_tree_attend";
    TreeArgs a{};
    int rc = tree_sizes(p->cfg, n_sessions, n_q_tokens, false, 0);
    if (rc == KVMEM_OK) rc = tree_common(p, n_sessions, q, n_q_tokens, n_q, mask, n_sel, tail, scale, out, lse, who, &a);
    if (rc != KVMEM_OK) return rc;
    if (!paged_block_size_ok(p, false, who)) return KVMEM_E_UNSUPPORTED;
    if (!sel_ids || sel_stride < 1 || (int64_t)sel_stride * p->cfg.block_tokens > INT32_MAX - 256) {
        set_error("kvmem_paged_tree_attend: sel_ids is null, or sel_stride is not positive or too long");
        return KVMEM_E_INVALID;
    }
    a.sel_ids = sel_ids; a.sel_stride = sel_stride; a.cap = sel_stride * p->cfg.block_tokens;
    a.pages = p->pages; a.tables = p->tables; a.nblocks_dev = p->nblocks_dev; a.session_first = session_first;
    a.max_bps = p->geo.max_bps; a.max_blocks = p->geo.max_blocks;
    return tree_run(p, a, workspace, workspace_bytes, stream, who);
}

int kvmem_view_attend_mass(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const int32_t* n_q,
                           const void* view_k, const void* view_v, int32_t view_cap_tokens, const int32_t* n_sel,
                           const kvmem_tail_t* tail, float scale, float* mass, float decay, void* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "kvmem_view_attend_mass";
    if (!pool_live(p)) return KVMEM_E_STATE;
    TreeArgs a{};
    int rc = tree_sizes(p->cfg, n_sessions, n_q_tokens, true, view_cap_tokens ? view_cap_tokens : -1);
    if (rc == KVMEM_OK) rc = tree_common(p, n_sessions, q, n_q_tokens, n_q, nullptr, n_sel, tail, scale, out, lse, who, &a);
    if (rc == KVMEM_OK) rc = tree_view(view_k, view_v, view_cap_tokens, who, &a);
    if (rc != KVMEM_OK) return rc;
    if (!mass || !aligned(mass, 16)) { set_error("kvmem_view_attend_mass: mass must be a 16-byte aligned device pointer"); return KVMEM_E_INVALID; }
    if (!(decay >= 0.0f) || !std::isfinite(decay)) { set_error("decay must be finite and non-negative"); return KVMEM_E_INVALID; }
    a.mass = mass; a.decay = decay;
    return tree_run(p, a, workspace, workspace_bytes, stream, who);
}

// What the eviction refuses for its size alone, and its workspace size with it; view_cap_tokens 0: a view of any length
static int evict_sizes(const kvmem_pool_config_t& c, int32_t n_sessions, int32_t keep_blocks, int32_t view_cap_tokens) {
    if (n_sessions < 1 || n_sessions > 65535) { set_error("n_sessions must be in [1, 65535]"); return KVMEM_E_INVALID; }
    if (keep_blocks < 1 || (int64_t)keep_blocks * c.block_tokens > INT32_MAX) { set_error("keep_blocks must be positive and keep_blocks * block_tokens below 2^31"); return KVMEM_E_INVALID; }
    if (c.head_dim != 128) { set_error("the eviction kernels are built for head_dim 128"); return KVMEM_E_UNSUPPORTED; }
    if (!evict_grid_fits(c, n_sessions, keep_blocks, view_cap_tokens)) {
        set_error("%d sessions with %d blocks kept are more than 2^31 pieces of 64 tokens, or 2^28 KV heads", n_sessions, keep_blocks);
        return KVMEM_E_UNSUPPORTED;
    }
    return KVMEM_OK;
}

size_t kvmem_evict_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t keep_blocks) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why)) { set_error("invalid arguments to kvmem_evict_workspace_bytes"); return 0; }
    if (evict_sizes(*cfg, n_sessions, keep_blocks, 0) != KVMEM_OK) return 0;
    return evict_workspace_bytes(*cfg, n_sessions, keep_blocks);
}

int kvmem_view_evict(kvmem_pool_t* p, int32_t n_sessions, const void* view_k, const void* view_v, int32_t view_cap_tokens,
                     const int32_t* n_sel, const float* mass, int32_t keep_blocks, int32_t n_sink_tokens, int32_t n_recent_tokens,
                     void* dst_k, void* dst_v, int32_t dst_cap_tokens, float* dst_mass, int32_t* kept, int32_t* n_sel_out,
                     void* workspace, size_t workspace_bytes, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    const int B = p->cfg.block_tokens;
    if (view_cap_tokens < B || view_cap_tokens % B != 0) { set_error("view_cap_tokens must be a positive multiple of block_tokens"); return KVMEM_E_INVALID; }
    const int rc = evict_sizes(p->cfg, n_sessions, keep_blocks, view_cap_tokens);
    if (rc != KVMEM_OK) return rc;
    if (!view_k || !view_v || !n_sel || !mass || !dst_k || !dst_v || !dst_mass || !n_sel_out || !workspace || !aligned(view_k, 128) ||
        !aligned(view_v, 128) || !aligned(dst_k, 128) || !aligned(dst_v, 128) || !aligned(mass, 16) || !aligned(dst_mass, 16) ||
        !aligned(workspace, 256)) {
        set_error("kvmem_view_evict: null or misaligned pointer (views need 128-byte alignment)");
        return KVMEM_E_INVALID;
    }
    if ((int64_t)keep_blocks * B > dst_cap_tokens) { set_error("the destination holds %d tokens, %d blocks are to be kept", dst_cap_tokens, keep_blocks); return KVMEM_E_INVALID; }
    if (n_sink_tokens < 0 || n_recent_tokens < 0) { set_error("n_sink_tokens and n_recent_tokens must not be negative"); return KVMEM_E_INVALID; }
    const size_t heads = (size_t)n_sessions * p->geo.L * p->geo.G;
    const size_t src_b = heads * view_cap_tokens * 256, dst_b = heads * dst_cap_tokens * 256;
    if (overlap(view_k, src_b, dst_k, dst_b) || overlap(view_k, src_b, dst_v, dst_b) || overlap(view_v, src_b, dst_k, dst_b) ||
        overlap(view_v, src_b, dst_v, dst_b) || overlap(dst_k, dst_b, dst_v, dst_b) ||
        overlap(mass, heads * view_cap_tokens * 4, dst_mass, heads * dst_cap_tokens * 4)) {
        set_error("kvmem_view_evict moves tokens out of place: source and destination overlap");
        return KVMEM_E_INVALID;
    }
    const size_t need = evict_workspace_bytes(p->cfg, n_sessions, keep_blocks);
    if (workspace_bytes < need) { set_error("evict workspace holds %zu bytes, %zu needed", workspace_bytes, need); return KVMEM_E_CAPACITY; }
    EvictArgs a{};
    a.view_k = (const __nv_bfloat16*)view_k; a.view_v = (const __nv_bfloat16*)view_v; a.n_sel = n_sel; a.mass = mass;
    a.dst_k = (__nv_bfloat16*)dst_k; a.dst_v = (__nv_bfloat16*)dst_v; a.dst_mass = dst_mass; a.kept = kept; a.n_sel_out = n_sel_out;
    a.ns = n_sessions; a.LG = p->geo.L * p->geo.G; a.B = B; a.cap = view_cap_tokens; a.dst_cap = dst_cap_tokens; a.keep = keep_blocks;
    a.n_sink = n_sink_tokens; a.n_recent = n_recent_tokens;
    cudaError_t e = launch_evict(*p, a, workspace, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("eviction kernel launch", e);
    return KVMEM_OK;
}

// ---- new tokens: rotary forms, tail and pages, prompt chunks ----

// form and frequencies of a rotary form; null: the pool's own
static int rope_form(const kvmem_pool_config_t& c, const kvmem_rope_t* r, RopeForm* form, double* f) {
    if (c.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    const kvmem_rope_t own{};
    if (!r) r = &own;
    const int d = c.head_dim, n = r->rotary_dim ? r->rotary_dim : d;
    if (r->layout != KVMEM_ROPE_HALF && r->layout != KVMEM_ROPE_INTERLEAVED) { set_error("layout must be KVMEM_ROPE_HALF or KVMEM_ROPE_INTERLEAVED"); return KVMEM_E_INVALID; }
    if (n < 0 || n > d) { set_error("rotary_dim %d outside [0, head_dim = %d]", n, d); return KVMEM_E_INVALID; }
    if (n % 16 != 0) { set_error("rotary_dim %d is not a multiple of 16", n); return KVMEM_E_UNSUPPORTED; }
    if (r->scaling < KVMEM_ROPE_NONE || r->scaling > KVMEM_ROPE_BANDS) { set_error("unknown scaling %d", r->scaling); return KVMEM_E_INVALID; }
    const bool scaled = r->scaling != KVMEM_ROPE_NONE, windowed = r->scaling == KVMEM_ROPE_RAMP || r->scaling == KVMEM_ROPE_BANDS;
    if (scaled && (!(r->factor >= 1.0f) || !std::isfinite(r->factor))) { set_error("factor must be finite and at least 1"); return KVMEM_E_INVALID; }
    const double factor = scaled ? (double)r->factor : 1.0, theta = (double)c.rope_theta, two_pi = 6.283185307179586476925286766559;
    const double fast = r->turns_fast != 0.0f ? (double)r->turns_fast : r->scaling == KVMEM_ROPE_RAMP ? 32.0 : 4.0;
    const double slow = r->turns_slow != 0.0f ? (double)r->turns_slow : 1.0, window = (double)r->original_positions;
    if (windowed && (!(window > 0.0) || !std::isfinite(window))) { set_error("original_positions must be positive and finite"); return KVMEM_E_INVALID; }
    if (windowed && (!(slow > 0.0) || !(fast > slow) || !std::isfinite(fast))) { set_error("turns_fast must be finite and exceed turns_slow, which must be positive"); return KVMEM_E_INVALID; }
    *form = RopeForm{n, n / 16, r->layout == KVMEM_ROPE_INTERLEAVED ? 1 : 0};
    auto pair_of = [&](double turns) { return n * log(window / (turns * two_pi)) / (2.0 * log(theta)); };
    const double lo = windowed ? std::max(floor(pair_of(fast)), 0.0) : 0.0, hi = windowed ? std::min(ceil(pair_of(slow)), n - 1.0) : 0.0;
    for (int i = 0; i < d / 2; ++i) {
        f[i] = 0.0;                                         // the dims that pass
        if (2 * i >= n) continue;
        f[i] = pow(theta, -2.0 * (double)i / (double)n);
        if (r->scaling == KVMEM_ROPE_LINEAR) f[i] /= factor;
        else if (r->scaling == KVMEM_ROPE_BASE) f[i] = pow(theta * pow(factor, n / (n - 2.0)), -2.0 * (double)i / (double)n);
        else if (windowed) {
            const double divided = r->scaling == KVMEM_ROPE_RAMP ? (i - lo) / std::max(hi - lo, 0.001)
                                                                 : (fast - window * f[i] / two_pi) / (fast - slow);
            const double x = std::min(std::max(divided, 0.0), 1.0);
            f[i] = f[i] / factor * x + f[i] * (1.0 - x);
        }
    }
    return KVMEM_OK;
}

int kvmem_rope_frequencies(const kvmem_pool_config_t* cfg, const kvmem_rope_t* rope, double* frequencies) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why) || !frequencies) { set_error("invalid arguments to kvmem_rope_frequencies: %s", why); return KVMEM_E_INVALID; }
    RopeForm form;
    double f[256];
    const int rc = rope_form(*cfg, rope, &form, f);
    if (rc == KVMEM_OK) memcpy(frequencies, f, sizeof(double) * (cfg->head_dim / 2));
    return rc;
}

// Calls that change what the host knows of a pool run once: a captured one would be replayed without the host's part.
static bool captured(void* stream, const char* who) {
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    const cudaError_t e = cudaStreamIsCapturing((cudaStream_t)stream, &st);
    if (e == cudaSuccess && st == cudaStreamCaptureStatusNone) return false;
    (void)cudaGetLastError();
    set_error("%s changes the pool's bookkeeping on the host: it cannot be part of a captured graph", who);
    return true;
}

int kvmem_set_rope(kvmem_pool_t* p, const kvmem_rope_t* rope, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (captured(stream, "kvmem_set_rope")) return KVMEM_E_STATE;
    RopeForm form;
    RopeFrequencies f{};
    const int rc = rope_form(p->cfg, rope, &form, f.f);
    if (rc != KVMEM_OK) return rc;
    for (int s = 0; s < p->cfg.max_sessions; ++s)
        if (p->sess_blocks[s] || !p->sess_reserved[s].empty()) {
            set_error("session %d holds blocks: the rotary form of a pool is set before tokens come in", s);
            return KVMEM_E_STATE;
        }
    // The pool's own frequencies give the table that it was created with, to the bit: where the device's 64-bit cosine and the host's differ in
    // their last bit, one entry in some 10^9 rounds to another fp32.
    double own[256];
    own_frequencies(p->cfg, own);
    if (memcmp(f.f, own, sizeof(double) * (p->cfg.head_dim / 2)) == 0) {
        if (!p->rope_own) {
            const int copied = upload_rope_table(*p, own, (cudaStream_t)stream);
            if (copied != KVMEM_OK) return copied;
            p->rope_own = true;
        }
    } else {
        p->rope_own = false;
        const cudaError_t e = launch_rope_table(*p, f, (cudaStream_t)stream);
        if (e != cudaSuccess) return cuda_fail("rotary table kernel launch", e);
    }
    p->rope_form = form;
    return KVMEM_OK;
}

static bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s < (1ll << 40); }

int kvmem_rope_apply(kvmem_pool_t* p, const void* x, int64_t x_row_stride, int64_t x_vec_stride, int32_t x_order, void* y,
                     int64_t y_row_stride, int64_t y_vec_stride, int32_t y_order, int64_t n_rows, int32_t n_vec,
                     const int32_t* positions, int32_t inverse, float amplitude, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (p->cfg.rope_max_positions <= 0) { set_error("the pool was created without rotary support"); return KVMEM_E_STATE; }
    if (n_rows < 0 || n_rows >= (1ll << 40) || n_vec < 1 || n_vec > (1 << 24)) { set_error("kvmem_rope_apply: n_rows must be in [0, 2^40), n_vec in [1, 2^24]"); return KVMEM_E_INVALID; }
    if ((x_order | 1) != 1 || (y_order | 1) != 1) { set_error("kvmem_rope_apply: an order is KVMEM_ORDER_MODEL or KVMEM_ORDER_POOL"); return KVMEM_E_INVALID; }
    if (!std::isfinite(amplitude) || amplitude < 0.0f) { set_error("amplitude must be finite and non-negative (0 selects 1)"); return KVMEM_E_INVALID; }
    if (n_rows == 0) return KVMEM_OK;
    if (n_rows == 1) x_row_stride = y_row_stride = 0;
    if (n_vec == 1) x_vec_stride = y_vec_stride = 0;
    if (!x || !y || !positions || !aligned(x, 16) || !aligned(y, 16) || !stride_ok(x_row_stride) || !stride_ok(x_vec_stride) ||
        !stride_ok(y_row_stride) || !stride_ok(y_vec_stride)) {
        set_error("kvmem_rope_apply: null or misaligned pointer, or a stride that is negative or no multiple of 8 elements");
        return KVMEM_E_INVALID;
    }
    const int64_t d = p->cfg.head_dim, rows1 = n_rows - 1, vec1 = n_vec - 1;
    // every element of y is written once
    const bool rows_outside = (vec1 == 0 || y_vec_stride >= d) && (rows1 == 0 || y_row_stride >= vec1 * y_vec_stride + d);
    const bool vecs_outside = (rows1 == 0 || y_row_stride >= d) && (vec1 == 0 || y_vec_stride >= rows1 * y_row_stride + d);
    if (!rows_outside && !vecs_outside) { set_error("kvmem_rope_apply: the strides of y make its vectors overlap"); return KVMEM_E_INVALID; }
    const size_t xb = 2 * (size_t)(rows1 * x_row_stride + vec1 * x_vec_stride + d), yb = 2 * (size_t)(rows1 * y_row_stride + vec1 * y_vec_stride + d);
    if (overlap(x, xb, y, yb)) {
        const RopeForm& f = p->rope_form;
        const bool same_order = x_order == y_order || (!f.interleaved && f.rotary == d);
        if (x != y || (rows1 && x_row_stride != y_row_stride) || (vec1 && x_vec_stride != y_vec_stride) || !same_order) {
            set_error("kvmem_rope_apply: x and y overlap without being the same vectors in the same order");
            return KVMEM_E_INVALID;
        }
    }
    RopeApplyArgs a{};
    a.x = (const __nv_bfloat16*)x; a.y = (__nv_bfloat16*)y; a.x_row = x_row_stride; a.x_vec = x_vec_stride; a.y_row = y_row_stride; a.y_vec = y_vec_stride;
    a.positions = positions; a.rope = p->rope_dev; a.status = p->status_dev; a.form = p->rope_form;
    a.n_vec = n_vec; a.d = p->cfg.head_dim; a.rope_positions = p->cfg.rope_max_positions; a.x_pool = x_order; a.y_pool = y_order;
    a.sgn = inverse ? -1.0f : 1.0f; a.amplitude = amplitude > 0.0f ? amplitude : 1.0f;
    const cudaError_t e = launch_rope_apply(*p, a, n_rows, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("rotary kernel launch", e);
    return KVMEM_OK;
}

int kvmem_rope_apply_call(const kvmem_rope_call_t* c) {
    if (!c) { set_error("null call"); return KVMEM_E_INVALID; }
    return kvmem_rope_apply(c->pool, c->x, c->x_row_stride, c->x_vec_stride, c->x_order, c->y, c->y_row_stride, c->y_vec_stride, c->y_order, c->n_rows,
                            c->n_vec, c->positions, c->inverse, c->amplitude, c->stream);
}

int kvmem_reserve_blocks(kvmem_pool_t* p, int32_t session, int32_t n_blocks, const int32_t* phys_ids, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    if (captured(stream, "kvmem_reserve_blocks") || !pages_are(p, false, "kvmem_reserve_blocks")) return KVMEM_E_STATE;
    if (p->cfg.rope_in_block_keys) { set_error("kvmem_reserve_blocks: reserved pages hold raw keys until they are indexed; the pool's pages hold keys rotated by their offset in the block"); return KVMEM_E_STATE; }
    if (n_blocks < 0) { set_error("n_blocks is negative"); return KVMEM_E_INVALID; }
    if (n_blocks == 0) return KVMEM_OK;
    std::vector<int32_t>& reserved = p->sess_reserved[session];
    const int64_t have = (int64_t)p->sess_blocks[session] + (int64_t)reserved.size();
    if (have + n_blocks > p->cfg.max_blocks_per_session) {
        set_error("session %d holds %lld blocks with the reserved ones; %d more exceed max_blocks_per_session = %d", session, (long long)have, n_blocks, p->cfg.max_blocks_per_session);
        return KVMEM_E_CAPACITY;
    }
    std::vector<int32_t> ids;
    try {
        ids.resize(n_blocks);
        const int rc = choose_pages(p, n_blocks, phys_ids, ids);
        if (rc != KVMEM_OK) return rc;
        reserved.reserve(reserved.size() + n_blocks);
    } catch (const std::bad_alloc&) { set_error("host allocation failed"); return KVMEM_E_CAPACITY; }
    const cudaError_t e = cudaMemcpyAsync(p->tables + (size_t)session * p->cfg.max_blocks_per_session + have, ids.data(), (size_t)n_blocks * 4,
                                          cudaMemcpyHostToDevice, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("block table upload", e);
    for (int32_t pg : ids) { p->page_used[pg] = 1; reserved.push_back(pg); }
    if (!phys_ids) p->free_hint = ids.back() + 1;
    return KVMEM_OK;
}

int32_t kvmem_session_reserved(const kvmem_pool_t* p, int32_t session) {
    if (!pool_ok(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    return (int32_t)p->sess_reserved[session].size();
}

// a tail whose rows are written, of n_sessions sessions and at least min_tokens tokens each
static int tail_ok(const kvmem_tail_t* tail, int32_t n_sessions, int32_t min_tokens, const char* who) {
    if (!tail || !tail->k || !tail->v || !tail->n_tokens || !aligned(tail->k, 16) || !aligned(tail->v, 16)) {
        set_error("%s: null or misaligned tail pointer", who);
        return KVMEM_E_INVALID;
    }
    if (tail->cap_tokens < min_tokens || tail->cap_tokens < 1 || (int64_t)tail->cap_tokens * n_sessions > INT32_MAX) {
        set_error("the tail holds %d tokens per session: at least %d are needed, and n_sessions * cap_tokens must stay below 2^31", tail->cap_tokens, min_tokens);
        return KVMEM_E_INVALID;
    }
    return KVMEM_OK;
}

// bytes from the first to behind the last element
static size_t rows_bytes(const kvmem_rows_t& r, int64_t ns, int64_t M, int64_t L, int64_t heads, int64_t d) {
    return 2 * (size_t)((ns - 1) * r.session_stride + (M - 1) * r.token_stride + (L - 1) * r.layer_stride + (heads - 1) * r.head_stride + d);
}

int kvmem_append_tokens(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, int32_t n_new_tokens, const int32_t* n_new,
                        const kvmem_rows_t* q, const kvmem_rows_t* k, const kvmem_rows_t* v, const int32_t* positions,
                        const int32_t* n_sel, int32_t first_position, float q_amplitude, const kvmem_tail_t* tail, void* q_out,
                        int32_t to_pages, void* stream) {
    const char* who = "kvmem_append_tokens";
    if (!pool_live(p)) return KVMEM_E_STATE;
    const Geometry& g = p->geo;
    if (n_sessions < 1 || n_sessions > 65535 || n_new_tokens < 1) { set_error("n_sessions must be in [1, 65535] and n_new_tokens positive"); return KVMEM_E_INVALID; }
    if (to_pages != 0 && to_pages != 1) { set_error("to_pages must be 0 or 1"); return KVMEM_E_INVALID; }
    if (to_pages) {
        if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
        if (!pages_are(p, false, who)) return KVMEM_E_STATE;
        if (p->cfg.rope_in_block_keys) { set_error("%s: pages that hold keys rotated by their offset in the block are filled by whole blocks", who); return KVMEM_E_STATE; }
    }
    if (g.d % 16 != 0) { set_error("%s needs head_dim to be a multiple of 16", who); return KVMEM_E_UNSUPPORTED; }
    if (!append_tokens_fits(p->cfg, n_new_tokens)) { set_error("%d new tokens per session are more than 2^31 groups of 16 elements: append them in parts", n_new_tokens); return KVMEM_E_UNSUPPORTED; }
    const int rc = tail_ok(tail, n_sessions, n_new_tokens, who);
    if (rc != KVMEM_OK) return rc;
    kvmem_rows_t copies[3];
    const kvmem_rows_t* in[3] = {q, k, v};
    for (int i = 0; i < 3; ++i) {                       // the stride of an axis of length 1 means nothing
        if (!in[i]) continue;
        copies[i] = *in[i];
        in[i] = &copies[i];
        if (n_sessions == 1) copies[i].session_stride = 0;
        if (n_new_tokens == 1) copies[i].token_stride = 0;
        if (g.L == 1) copies[i].layer_stride = 0;
        if ((i ? g.G : g.H) == 1) copies[i].head_stride = 0;
    }
    if (!k || !v || !q != !q_out || !aligned(q_out, 16)) { set_error("%s: k and v are required, q and q_out go together and are 16-byte aligned", who); return KVMEM_E_INVALID; }
    for (const kvmem_rows_t* r : in)
        if (r && (!r->data || !aligned(r->data, 16) || !stride_ok(r->session_stride) || !stride_ok(r->token_stride) || !stride_ok(r->layer_stride) || !stride_ok(r->head_stride))) {
            set_error("%s: null or misaligned rows, or a stride that is negative or no multiple of 8 elements", who);
            return KVMEM_E_INVALID;
        }
    for (int i = 0; i < 3; ++i)
        if (in[i] && (g.L - 1) * in[i]->layer_stride + ((i ? g.G : g.H) - 1) * in[i]->head_stride >= (1ll << 31)) {
            set_error("%s: the layers and heads of a token lie more than 2^31 elements apart", who);
            return KVMEM_E_UNSUPPORTED;
        }
    if (!std::isfinite(q_amplitude) || q_amplitude < 0.0f) { set_error("q_amplitude must be finite and non-negative (0 selects 1)"); return KVMEM_E_INVALID; }
    const bool rope = p->cfg.rope_max_positions > 0;
    if (rope && !positions && (first_position < 0 || first_position >= p->cfg.rope_max_positions)) {
        set_error("first_position %d outside the rotary table [0, %d)", first_position, p->cfg.rope_max_positions);
        return KVMEM_E_INVALID;
    }
    const size_t tail_b = 2 * (size_t)n_sessions * tail->cap_tokens * g.L * g.G * g.d, q_b = 2 * (size_t)n_sessions * n_new_tokens * g.L * g.H * g.d;
    const void* outs[3] = {tail->k, tail->v, q_out};
    const size_t out_b[3] = {tail_b, tail_b, q_b};
    for (int i = 0; i < 3; ++i) {
        if (!outs[i]) continue;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], out_b[i], outs[j], out_b[j])) { set_error("%s: two of tail.k, tail.v and q_out overlap", who); return KVMEM_E_INVALID; }
        for (int j = 0; j < 3; ++j)
            if (in[j] && overlap(outs[i], out_b[i], in[j]->data, rows_bytes(*in[j], n_sessions, n_new_tokens, g.L, j ? g.G : g.H, g.d))) {
                set_error("%s: a result overlaps q, k or v", who);
                return KVMEM_E_INVALID;
            }
    }
    AppendTokensArgs a{};
    auto rows = [](const kvmem_rows_t* r) { return r ? TokenRows{(const __nv_bfloat16*)r->data, r->session_stride, r->token_stride, (int)r->layer_stride, (int)r->head_stride} : TokenRows{}; };
    a.q = rows(in[0]); a.k = rows(in[1]); a.v = rows(in[2]);
    a.q_out = (__nv_bfloat16*)q_out; a.tail_k = (__nv_bfloat16*)tail->k; a.tail_v = (__nv_bfloat16*)tail->v;
    a.tail_n = tail->n_tokens; a.n_new = n_new; a.positions = positions; a.n_sel = n_sel;
    a.rope = rope ? p->rope_dev : nullptr; a.pages = to_pages ? p->pages : nullptr; a.tables = p->tables; a.nblocks_dev = p->nblocks_dev;
    a.status = p->status_dev; a.page_elems = p->lay.page_elems; a.form = p->rope_form;
    if (!rope) a.form.chunks = 0;
    a.ns = n_sessions; a.M = n_new_tokens; a.L = g.L; a.Hq = q ? g.H : 0; a.G = g.G; a.d = g.d; a.B = g.B; a.tail_cap = tail->cap_tokens;
    a.first_position = first_position; a.rope_positions = p->cfg.rope_max_positions; a.session_first = session_first; a.max_bps = g.max_bps;
    a.max_blocks = g.max_blocks; a.q_amplitude = q_amplitude > 0.0f ? q_amplitude : 1.0f;
    const cudaError_t e = launch_append_tokens(*p, a, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail("token append kernel launch", e);
    return KVMEM_OK;
}

int kvmem_append_tokens_call(const kvmem_append_call_t* c) {
    if (!c) { set_error("null call"); return KVMEM_E_INVALID; }
    return kvmem_append_tokens(c->pool, c->session_first, c->n_sessions, c->n_new_tokens, c->n_new, c->q.data ? &c->q : nullptr, &c->k, &c->v, c->positions,
                               c->n_sel, c->first_position, c->q_amplitude, &c->tail, c->q_out, c->to_pages, c->stream);
}

int kvmem_commit_blocks(kvmem_pool_t* p, int32_t session_first, int32_t n_sessions, const int32_t* n_blocks, const kvmem_tail_t* tail, void* stream) {
    const char* who = "kvmem_commit_blocks";
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session_first, n_sessions)) return KVMEM_E_INVALID;
    if (!n_blocks) { set_error("%s: n_blocks is null", who); return KVMEM_E_INVALID; }
    if (captured(stream, who)) return KVMEM_E_STATE;
    if (tail) {
        const int rc = tail_ok(tail, n_sessions, 1, who);
        if (rc != KVMEM_OK) return rc;
    }
    for (int i = 0; i < n_sessions; ++i) {
        const size_t reserved = p->sess_reserved[session_first + i].size();
        if (n_blocks[i] < 0) { set_error("n_blocks[%d] is negative", i); return KVMEM_E_INVALID; }
        if ((size_t)n_blocks[i] > reserved) { set_error("session %d has %zu reserved blocks, %d are to be committed", session_first + i, reserved, n_blocks[i]); return KVMEM_E_STATE; }
    }
    const Geometry& g = p->geo;
    try {
        for (int i = 0; i < n_sessions; ++i)
            if (n_blocks[i]) p->sess_pages[session_first + i].reserve(p->sess_pages[session_first + i].size() + n_blocks[i]);
    } catch (const std::bad_alloc&) { set_error("host allocation failed"); return KVMEM_E_CAPACITY; }
    for (int i0 = 0; i0 < n_sessions;) {
        CommitArgs a{};
        int i = i0;
        for (; i < n_sessions && a.ns < kCommitSessions; ++i)
            if (n_blocks[i]) a.s[a.ns++] = CommitSession{session_first + i, i, p->sess_blocks[session_first + i], n_blocks[i]};
        i0 = i;
        if (a.ns == 0) break;
        a.pages = p->pages; a.index = p->index; a.tables = p->tables; a.nblocks = p->nblocks_dev; a.status = p->status_dev;
        a.page_elems = p->lay.page_elems; a.index_elems = p->lay.index_elems_per_session;
        a.L = g.L; a.G = g.G; a.d = g.d; a.B = g.B; a.max_bps = g.max_bps; a.max_blocks = g.max_blocks;
        if (tail) { a.tail_n = const_cast<int32_t*>(tail->n_tokens); a.tail_k = (__nv_bfloat16*)tail->k; a.tail_v = (__nv_bfloat16*)tail->v; a.tail_cap = tail->cap_tokens; }
        const cudaError_t e = launch_commit(a, (cudaStream_t)stream);
        if (e != cudaSuccess) return cuda_fail("block commit kernel launch", e);
        for (int k = 0; k < a.ns; ++k) {
            std::vector<int32_t>&reserved = p->sess_reserved[a.s[k].session], &pages = p->sess_pages[a.s[k].session];
            pages.insert(pages.end(), reserved.begin(), reserved.begin() + a.s[k].n);
            reserved.erase(reserved.begin(), reserved.begin() + a.s[k].n);
            p->sess_blocks[a.s[k].session] += a.s[k].n;
        }
    }
    return KVMEM_OK;
}

int kvmem_get_pages(kvmem_pool_t* p, const void** pages) {
    if (!pool_ok(p)) return KVMEM_E_STATE;
    if (!pages) { set_error("null output pointer"); return KVMEM_E_INVALID; }
    *pages = p->pages;
    return KVMEM_OK;
}

// What the chunk attention refuses for its size alone, and its workspace size with it; capacities 0: any
static int prefill_sizes(const kvmem_pool_config_t& c, int32_t n_sessions, int32_t n_q_tokens, int32_t cap, int32_t tail_cap) {
    if (n_sessions < 1 || n_sessions > 65535) { set_error("n_sessions must be in [1, 65535]"); return KVMEM_E_INVALID; }
    if (n_q_tokens < 1) { set_error("n_q_tokens must be positive"); return KVMEM_E_INVALID; }
    if (c.head_dim != 128) { set_error("the attention kernel is built for head_dim 128"); return KVMEM_E_UNSUPPORTED; }
    if (c.n_q_heads / c.n_kv_heads > 128) { set_error("more than 128 query heads share a KV head"); return KVMEM_E_UNSUPPORTED; }
    if (!prefill_fits(c, n_sessions, n_q_tokens, cap, tail_cap)) {
        set_error("%d sessions of %d new tokens over up to %d + %d tokens are more than a line of 2^30 tiles", n_sessions, n_q_tokens, cap, tail_cap);
        return KVMEM_E_UNSUPPORTED;
    }
    return KVMEM_OK;
}

// A chunk of up to 64 tokens is a chain of drafted ones, and where its query rows are few the decode kernel is faster: it shares a tile's
// two slots out between tokens.  With more rows the chunk's own kernel is.  Measured, 64-token blocks, tail of 40, us at 2,048 / 16,384 /
// 65,536 tokens, decode kernel and chunk kernel:
//   64 heads on 8, 48 tokens (384 rows a KV head, 3,072 in all)     24 / 43 / 129    23 / 47 / 131
//   64 heads on 8, 64 tokens (512 and 4,096)                        25 / 51 / 170    25 / 50 / 143
//   64 heads on 4, 33 tokens (528 and 2,112)                        25 / 37 / 102    26 / 40 / 108
//   64 heads on 4, 64 tokens (1,024 and 4,096)                      25 / 51 / 179    25 / 47 / 137
//   128 heads on 4, 16 tokens (512 and 2,048)                       23 / 34 / 80     29 / 38 / 80
//   128 heads on 4, 24 tokens (768 and 3,072)                       26 / 44 / 120    26 / 42 / 108
//   32 heads on 8, 64 tokens (256 and 2,048), 2,048 / 32,768        20 / 50          26 / 57
static bool chunk_is_chain(const kvmem_pool_config_t& c, int32_t n_sessions, int32_t n_q_tokens) {
    if (n_q_tokens < 1 || n_q_tokens > kMaxDrafted) return false;
    const int64_t share = c.n_q_heads / c.n_kv_heads, rows = (int64_t)n_sessions * c.n_layers * c.n_q_heads * n_q_tokens;
    return share > 128 || share * n_q_tokens < 448 || rows < 2560;
}

size_t kvmem_prefill_workspace_bytes(const kvmem_pool_config_t* cfg, int32_t n_sessions, int32_t n_q_tokens) {
    const char* why = "";
    if (!cfg || !config_valid(*cfg, &why)) { set_error("invalid arguments to kvmem_prefill_workspace_bytes"); return 0; }
    if (chunk_is_chain(*cfg, n_sessions, n_q_tokens)) return tree_bytes(cfg, n_sessions, n_q_tokens, 0, "kvmem_prefill_workspace_bytes");
    if (prefill_sizes(*cfg, n_sessions, n_q_tokens, 0, 0) != KVMEM_OK) return 0;
    return prefill_workspace_bytes(*cfg);
}

int kvmem_view_prefill_attend(kvmem_pool_t* p, int32_t n_sessions, const void* q, int32_t n_q_tokens, const int32_t* n_q,
                              const void* view_k, const void* view_v, int32_t view_cap_tokens, const int32_t* n_sel,
                              const kvmem_tail_t* tail, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                              void* stream) {
    const char* who = "kvmem_view_prefill_attend";
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (chunk_is_chain(p->cfg, n_sessions, n_q_tokens))
        return kvmem_view_tree_attend(p, n_sessions, q, n_q_tokens, n_q, nullptr, view_k, view_v, view_cap_tokens, n_sel, tail, scale, out, lse, workspace,
                                      workspace_bytes, stream);
    const Geometry& g = p->geo;
    if (view_cap_tokens < g.B || view_cap_tokens % g.B != 0) { set_error("view_cap_tokens must be a positive multiple of block_tokens"); return KVMEM_E_INVALID; }
    int rc = KVMEM_OK;
    if (tail && n_sessions >= 1) rc = tail_ok(tail, n_sessions, n_q_tokens, who);
    if (rc == KVMEM_OK) rc = prefill_sizes(p->cfg, n_sessions, n_q_tokens, view_cap_tokens, tail ? tail->cap_tokens : 0);
    if (rc != KVMEM_OK) return rc;
    if (!q || !view_k || !view_v || !n_sel || !out || !lse || !workspace || !aligned(q, 16) || !aligned(view_k, 128) || !aligned(view_v, 128) ||
        !aligned(out, 16) || !aligned(workspace, 256)) {
        set_error("%s: null or misaligned pointer (views need 128-byte alignment)", who);
        return KVMEM_E_INVALID;
    }
    if (!(scale >= 0.0f) || !std::isfinite(scale)) { set_error("scale must be finite and non-negative (0 selects 1/sqrt(d))"); return KVMEM_E_INVALID; }
    const size_t need = prefill_workspace_bytes(p->cfg);
    if (workspace_bytes < need) { set_error("%s: the workspace holds %zu bytes, %zu needed", who, workspace_bytes, need); return KVMEM_E_CAPACITY; }
    PrefillArgs a{};
    a.q = (const __nv_bfloat16*)q; a.n_q = n_q; a.view_k = (const __nv_bfloat16*)view_k; a.view_v = (const __nv_bfloat16*)view_v; a.n_sel = n_sel;
    if (tail) { a.tail_k = (const __nv_bfloat16*)tail->k; a.tail_v = (const __nv_bfloat16*)tail->v; a.n_tail = tail->n_tokens; a.tail_cap = tail->cap_tokens; }
    a.out = (__nv_bfloat16*)out; a.lse = lse; a.status = p->status_dev;
    a.ns = n_sessions; a.M = n_q_tokens; a.L = g.L; a.H = g.H; a.G = g.G; a.r = g.r; a.B = g.B; a.cap = view_cap_tokens;
    a.scale = scale > 0.0f ? scale : 1.0f / sqrtf((float)g.d);
    const cudaError_t e = launch_prefill(*p, a, workspace, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(who, e);
    return KVMEM_OK;
}

int kvmem_get_index(kvmem_pool_t* p, int32_t session, const void** index, int32_t* n_blocks) {
    if (!pool_ok(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    if (!index || !n_blocks) { set_error("null output pointer"); return KVMEM_E_INVALID; }
    *index = p->index + (size_t)session * p->lay.index_elems_per_session;
    *n_blocks = p->sess_blocks[session];
    return KVMEM_OK;
}

int kvmem_get_block_table(kvmem_pool_t* p, int32_t session, const int32_t** table, int32_t* n_blocks) {
    if (!pool_ok(p)) return KVMEM_E_STATE;
    if (!sessions_ok(p, session, 1)) return KVMEM_E_INVALID;
    if (!table || !n_blocks) { set_error("null output pointer"); return KVMEM_E_INVALID; }
    *table = p->tables + (size_t)session * p->cfg.max_blocks_per_session;
    *n_blocks = p->sess_blocks[session];
    return KVMEM_OK;
}

int kvmem_device_status(kvmem_pool_t* p, int32_t* status, void* stream) {
    if (!pool_live(p)) return KVMEM_E_STATE;
    if (!status) { set_error("status is null"); return KVMEM_E_INVALID; }
    cudaStream_t st = (cudaStream_t)stream;
    int32_t word = 0;
    cudaError_t e = cudaMemcpyAsync(&word, p->status_dev, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(p->status_dev, 0, 4, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return cuda_fail("reading the device status word", e);
    *status = word;
    return KVMEM_OK;
}

}  // extern "C"
