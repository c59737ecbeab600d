"""Eviction by accumulated weight against a plain restatement (exact: nothing is rounded), and the decode loop that uses
attention, weights and eviction together."""
import math

import pytest
import torch

from kvmem_harness import Guards
from paper_2609_04852_b200 import KvmemError, Pool, Tail, View
from paper_2609_04852_b200 import kvmem

pytestmark = pytest.mark.gpu
D = 128


def reference_kept(mass, T, C, n_sink, n_recent):
    """Ascending kept tokens of one head; mass: a list of T floats."""
    K = min(C, T)
    sinks = min(n_sink, K)
    recents = min(n_recent, K - sinks)
    hold = set(range(sinks)) | set(range(T - recents, T))
    order = sorted((t for t in range(sinks, T - recents)), key=lambda t: (-math.inf if math.isnan(mass[t]) else 0, 0.0 if math.isnan(mass[t]) else -mass[t], t))
    return sorted(hold | set(order[:K - len(hold)]))


class Case:
    def __init__(self, ns=1, L=1, G=2, B=64, lens=(8,), keep=4, sink=0, recent=0, cap=None, dst_cap=None, kind="random", seed=0):
        dev = torch.device("cuda", torch.cuda.current_device())
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ns, self.L, self.G, self.B, self.lens, self.keep, self.sink, self.recent = ns, L, G, B, list(lens), keep, sink, recent
        self.cap = (max(max(lens), 1) + 1) * B if cap is None else cap
        self.dcap = keep * B + 2 * B if dst_cap is None else dst_cap
        self.k, self.v = (torch.randn(ns, L, G, self.cap, D, generator=gen, device=dev).to(torch.bfloat16) for _ in range(2))
        m = torch.rand(ns, L, G, self.cap, generator=gen, device=dev)
        if kind == "ties":
            m = (m * 4).floor() / 4
        elif kind == "zero":
            m = torch.zeros_like(m)
        elif kind == "heavy":
            m = torch.exp(6 * torch.randn(m.shape, generator=gen, device=dev))
        elif kind == "special":
            pick = torch.randint(0, 9, m.shape, generator=gen, device=dev)
            table = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1.0, 3.0, 1e38], device=dev)
            m = table[pick]
        self.mass = m
        self.n_sel = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.pool = Pool(L, 2 * G, G, D, B, ns, 1, 1, dev.index)
        self.guards = Guards(dev)
        sh = (ns, L, G, self.dcap)
        self.dst = View(self.guards.empty((*sh, D), torch.bfloat16, fill=5.0), self.guards.empty((*sh, D), torch.bfloat16, fill=6.0), self.dcap)
        self.dmass = self.guards.empty(sh, torch.float32, fill=7.0)
        self.kept = self.guards.empty((ns, L, G, keep * B), torch.int32, fill=-9)
        self.n_out = self.guards.empty((ns,), torch.int32, fill=-1)

    def call(self, **kw):
        args = dict(kept=self.kept, keep_blocks=self.keep, n_sink_tokens=self.sink, n_recent_tokens=self.recent)
        args.update(kw)
        self.pool.view_evict(View(self.k, self.v, self.cap), self.n_sel, self.mass, self.dst, self.n_out, self.dmass, **args)

    def check(self, kept_written=True):
        torch.cuda.synchronize()
        mass = self.mass.cpu()
        for s in range(self.ns):
            T = min(max(self.lens[s], 0) * self.B, self.cap)
            K = min(self.keep * self.B, T)
            assert int(self.n_out[s]) == K // self.B
            for l in range(self.L):
                for g in range(self.G):
                    want = torch.tensor(reference_kept(mass[s, l, g, :T].tolist(), T, self.keep * self.B, self.sink, self.recent), dtype=torch.int64)
                    assert len(want) == K
                    if kept_written:
                        assert torch.equal(self.kept[s, l, g, :K].cpu().long(), want), (s, l, g)
                        assert bool((self.kept[s, l, g, K:] == -9).all())
                    w = want.cuda()
                    assert torch.equal(self.dst.k[s, l, g, :K], self.k[s, l, g, w]) and torch.equal(self.dst.v[s, l, g, :K], self.v[s, l, g, w])
                    assert torch.equal(self.dmass[s, l, g, :K].view(torch.int32), self.mass[s, l, g, w].view(torch.int32))
                    assert bool((self.dst.k[s, l, g, K:] == 5.0).all()) and bool((self.dst.v[s, l, g, K:] == 6.0).all())
                    assert bool((self.dmass[s, l, g, K:] == 7.0).all())
        self.guards.check()


CASES = [
    dict(),
    dict(lens=(1,), keep=1),                                           # everything stays
    dict(lens=(3,), keep=9),                                           # room for more than there is
    dict(lens=(5,), keep=1, sink=64),                                  # the sinks alone
    dict(lens=(5,), keep=1, sink=100, recent=100),                     # more reserved than kept: sinks first
    dict(lens=(5,), keep=2, sink=10, recent=90),
    dict(lens=(5,), keep=2, sink=3, recent=1000),                      # recents fill what the sinks leave
    dict(lens=(5,), keep=2, sink=64, recent=64),                       # nothing is left for the weights
    dict(lens=(6,), keep=3, kind="ties", sink=1, recent=1),
    dict(lens=(6,), keep=3, kind="zero"),                              # all weights equal: the lowest tokens
    dict(lens=(6,), keep=3, kind="special", recent=5),
    dict(lens=(9,), keep=4, kind="heavy", B=16),
    dict(ns=3, L=2, lens=(4, 0, 11), keep=5, B=32, sink=7, recent=13, kind="ties"),
    dict(ns=4, G=1, lens=(40, 1, 17, 39), keep=16, B=128, kind="heavy"),
    dict(lens=(70,), keep=33, B=48, G=3, kind="ties"),
    dict(lens=(130,), keep=100, B=256, G=1, kind="heavy", recent=300),  # 33,280 tokens
    dict(lens=(640,), keep=77, G=1, kind="ties", sink=4),               # 40,960 tokens, a quarter of them at the bar
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_eviction_matches_the_definition(i):
    c = Case(seed=i, **CASES[i])
    c.call()
    c.check()


def test_without_the_list_of_kept_tokens():
    c = Case(lens=(7,), keep=3, seed=4)
    c.call(kept=None)
    c.check(kept_written=False)
    assert bool((c.kept == -9).all())


def test_lengths_out_of_range_are_clamped_and_the_length_may_be_updated_in_place():
    c = Case(ns=2, lens=(8, 8), keep=3, cap=8 * 64)
    c.n_sel[0], c.n_sel[1] = 1 << 30, -4
    c.lens = [8, -4]
    c.n_out = c.n_sel
    c.call()
    c.check()


def test_with_plain_launches():
    c = Case(ns=2, lens=(70, 9), keep=8, kind="ties", sink=3, seed=12)
    kvmem.set_option("pdl", 0)
    try:
        c.call()
        c.check()
    finally:
        kvmem.set_option("pdl", 1)


def test_two_streams_with_their_own_workspaces():
    cases = [Case(lens=(130,), keep=40, kind=kind, recent=5, seed=20 + i) for i, kind in enumerate(("heavy", "ties"))]
    need = [c.pool.lib.kvmem_evict_workspace_bytes(kvmem.C.byref(c.pool.cfg), c.ns, c.keep) for c in cases]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in need]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, w, st in zip(cases, ws, streams):
            with torch.cuda.stream(st):
                c.call(workspace=w, kept=None)
    for c in cases:
        c.check(kept_written=False)


def test_captured_eviction_follows_the_device():
    c = Case(ns=2, lens=(9, 4), keep=3, recent=20, seed=9)
    c.call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call()
    for lens in ((2, 10), (10, 0)):
        c.lens = list(lens)
        c.n_sel.copy_(torch.tensor(lens))
        c.mass.copy_(c.mass.flip(3))
        c.dst.k.fill_(5.0); c.dst.v.fill_(6.0); c.dmass.fill_(7.0); c.kept.fill_(-9)
        g.replay()
        c.check()


def test_a_native_window_and_offsets_past_32_bits():
    """Nine sessions of 262,144 tokens on 8 KV heads: more than 2^31 elements in the view; the last one is evicted."""
    ns, G, cap, keep = 9, 8, 262144, 1024
    dev = torch.device("cuda", 0)
    pool = Pool(1, 32, G, D, 64, ns, 1, 1, 0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.empty(ns, 1, G, cap, D, dtype=torch.bfloat16, device=dev)
    k[ns - 1] = torch.randn(1, G, cap, D, generator=gen, device=dev)
    v = -k
    mass = torch.rand(ns, 1, G, cap, generator=gen, device=dev)
    n_sel = torch.zeros(ns, dtype=torch.int32, device=dev)
    n_sel[ns - 1] = 4096
    dst = View(torch.zeros(ns, 1, G, keep * 64, D, dtype=torch.bfloat16, device=dev), torch.zeros(ns, 1, G, keep * 64, D, dtype=torch.bfloat16, device=dev), keep * 64)
    dm, kept = torch.zeros(ns, 1, G, keep * 64, device=dev), torch.zeros(ns, 1, G, keep * 64, dtype=torch.int32, device=dev)
    pool.view_evict(View(k, v, cap), n_sel, mass, dst, n_sel, dm, kept=kept, n_sink_tokens=3, n_recent_tokens=700)
    torch.cuda.synchronize()
    assert n_sel.tolist() == [0] * (ns - 1) + [keep]
    s = ns - 1
    for g in range(G):
        m = mass[s, 0, g].double()
        m[:3] = math.inf
        m[cap - 700:] = math.inf
        want = torch.argsort(-m, stable=True)[:keep * 64].sort().values
        assert torch.equal(kept[s, 0, g].long(), want)
        assert torch.equal(dst.k[s, 0, g], k[s, 0, g, want]) and torch.equal(dst.v[s, 0, g], v[s, 0, g, want])
        assert torch.equal(dm[s, 0, g], mass[s, 0, g, want])
    assert bool((dst.k[:s] == 0).all())


def test_refusals():
    c = Case()

    def raises(status, **kw):
        with pytest.raises(KvmemError) as e:
            c.call(**kw)
        assert e.value.status == status

    raises(kvmem.E_INVALID, n_sink_tokens=-1)
    raises(kvmem.E_INVALID, n_recent_tokens=-1)
    raises(kvmem.E_INVALID, keep_blocks=0, kept=None)
    raises(kvmem.E_INVALID, keep_blocks=7, kept=None)          # the destination holds six
    raises(kvmem.E_CAPACITY, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        c.call(kept=c.kept.long())
    dst, dm = c.dst, c.dmass
    c.dst, c.dmass = View(c.k, c.v, c.cap), torch.zeros_like(c.mass)
    raises(kvmem.E_INVALID)                                     # in place
    c.dst, c.dmass = View(torch.zeros_like(c.k), torch.zeros_like(c.k), c.cap), c.mass
    raises(kvmem.E_INVALID)                                     # the weights in place
    c.dst, c.dmass = dst, dm
    torch.cuda.synchronize()
    assert bool((c.dst.k == 5.0).all()) and bool((c.n_out == -1).all())


def test_decode_loop_with_drafts_weights_and_eviction():
    """Select, materialise, decode with weights, evict, then verify a draft tree over the smaller view: every step's input
    is the one before's output, and the end is compared with a plain run of the same loop in 64 bits."""
    from kvmem_harness import fill_pool, queries
    from kvmem_workloads import CONFIGS
    from paper_2609_04852_b200 import SelectParams
    spec = CONFIGS["tiny"].with_(n_blocks=64, n_planted=4, budget_blocks=12)
    pool = fill_pool(spec)
    dev, B, G, H, r = torch.device("cuda", 0), 64, 8, 32, 4
    q0, _ = queries(spec)
    q0 = q0.to(dev)
    sel, n_sel = torch.zeros(1, 12, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    pool.select(q0, SelectParams(12, spec.max_view_tokens, 0, 0, 0), sel, n_sel)
    view = pool.new_view(1, 12 * B)
    pool.materialize(sel, n_sel, view)
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=dev).to(torch.bfloat16)   # noqa: E731
    M = 6
    tail = Tail(rnd(1, 20, 1, G, D), rnd(1, 20, 1, G, D), torch.zeros(1, dtype=torch.int32, device=dev))
    mass = torch.zeros(1, 1, G, 12 * B, device=dev)
    qs = [rnd(1, 1, 1, H, D) for _ in range(4)]
    for i, q in enumerate(qs):                                   # four decoded tokens join the tail one by one
        out, lse = torch.zeros(1, 1, 1, H, D, dtype=torch.bfloat16, device=dev), torch.zeros(1, 1, 1, H, device=dev)
        tail.n_tokens.fill_(i)
        pool.view_attend_mass(q, view, n_sel, mass, out, lse, tail=tail, decay=0.8)
    small = pool.new_view(1, 5 * B)
    smass, sn = torch.zeros(1, 1, G, 5 * B, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    kept = torch.zeros(1, 1, G, 5 * B, dtype=torch.int32, device=dev)
    pool.view_evict(view, n_sel, mass, small, sn, smass, kept=kept, n_sink_tokens=2, n_recent_tokens=B)
    tail.n_tokens.fill_(4)
    qt = rnd(1, M, 1, H, D)
    rows = [[1, 3, 5, 11, 19, 33]]
    out, lse = torch.zeros(1, M, 1, H, D, dtype=torch.bfloat16, device=dev), torch.zeros(1, M, 1, H, device=dev)
    pool.view_tree_attend(qt, small, sn, tail, out, lse, mask=torch.tensor(rows, device=dev))
    torch.cuda.synchronize()
    assert pool.device_status() == 0 and sn.item() == 5 and n_sel.item() == 12
    # the view_attend of the framework reads the evicted view as any other
    o2, l2 = pool.new_outputs(1, M)
    pool.view_attend(qt, small, sn, o2, l2)
    o3, l3 = torch.zeros_like(out), torch.zeros_like(lse)
    pool.view_tree_attend(qt, small, sn, None, o3, l3)
    torch.cuda.synchronize()
    assert bool(((l2 - l3).abs() <= 1e-4).all()) and bool(((o2 - o3.float()).abs() <= 2.0 ** -7 * o2.abs() + 2e-3).all())
    for g in range(G):
        K, V = view.k[0, 0, g].double(), view.v[0, 0, g].double()
        tk, tv = tail.k[0, :, 0, g].double(), tail.v[0, :, 0, g].double()
        m = torch.zeros(12 * B, dtype=torch.float64, device=dev)
        for i, q in enumerate(qs):
            x = q[0, 0, 0, g * r:(g + 1) * r].double() @ torch.cat([K, tk[:i + 1]]).T / math.sqrt(D)
            m = 0.8 * m + x.softmax(1)[:, :12 * B].sum(0)
        # weights: sums of four steps whose relative error is below 1e-3 (logits of some 20 magnitudes at 2^-16 each)
        assert bool(((mass[0, 0, g].double() - m).abs() <= 1e-3 * m).all())
        ids = kept[0, 0, g].long()
        want = torch.tensor(reference_kept(mass[0, 0, g].tolist(), 12 * B, 5 * B, 2, B), device=dev)
        assert torch.equal(ids, want) and torch.equal(smass[0, 0, g], mass[0, 0, g, ids])
        Kt, Vt = torch.cat([K[ids], tk[:4 + M]]), torch.cat([V[ids], tv[:4 + M]])
        for i in range(M):
            see = torch.ones(5 * B + 4 + M, dtype=torch.bool)
            for j in range(M):
                see[5 * B + 4 + j] = bool((rows[0][i] >> j) & 1)
            see = see.to(dev)
            x = torch.where(see, qt[0, i, 0, g * r:(g + 1) * r].double() @ Kt.T / math.sqrt(D), -math.inf)
            p = x.softmax(1)
            ref = p @ Vt
            tol = (2.0 ** -8 + 2.0 ** -12) * (p @ Vt.abs()) + 2.0 ** -7 * ref.abs()
            assert bool(((out[0, i, 0, g * r:(g + 1) * r].double() - ref).abs() <= tol).all())
