"""Decode over a view at the edges of its definitions: infinities and NaN in the call that accumulates weights, both sides of
each choice of its last kernel, a wait of the attention kernel that runs out, the pool's own workspace, pools with rotary support."""
import gc
import math

import pytest
import torch

from paper_2609_04852_b200 import KvmemError, Pool
from paper_2609_04852_b200 import kvmem
from test_gpu_evict import Case as EvictCase
from test_gpu_tree import Case

pytestmark = pytest.mark.gpu


def weights_case(mass_seed=5, **kw):
    c = Case(mask="chain", **kw)
    c.mass = c.guards.empty((c.ns, c.L, c.G, c.capb * c.B), torch.float32)
    c.mass.copy_(torch.rand(c.mass.shape, generator=torch.Generator().manual_seed(mass_seed)))
    return c


RAGGED = dict(ns=2, L=2, lens=(3, 20), M=2, tails=(4, 0), seed=71)


@pytest.mark.parametrize("decay", [1.0, 0.5])
def test_rows_whose_logits_are_all_minus_infinity_add_nothing_to_the_weights(decay):
    """Everything that the rows of one KV head see has a key of -inf in a dimension where the queries are positive: out = 0
    (a drafted value that is not finite included), lse = -inf and the weights only decay; every other head is what it is
    without that.  The next step's weights are ordinary."""
    c, clean = weights_case(**RAGGED), weights_case(**RAGGED)
    s, l, g, r = 0, 1, 1, c.H // c.G
    heads = slice(g * r, (g + 1) * r)
    for x in (c, clean):
        x.q[s, :, l, heads, 5] = 1.5
    before, finite = c.mass.clone(), (c.k[s, l, g, :, 5].clone(), c.tk[s, :, l, g, 5].clone(), c.tv[s, c.tails[s], l, g, 9].clone())
    c.k[s, l, g, :, 5] = -math.inf
    c.tk[s, :, l, g, 5] = -math.inf
    c.tv[s, c.tails[s], l, g, 9] = math.inf
    c.call(decay=decay)
    clean.call(decay=decay)
    torch.cuda.synchronize()
    assert bool((c.out[s, :, l, heads] == 0).all()) and bool((c.lse[s, :, l, heads] == -math.inf).all())
    T = c.lens[s] * c.B
    want = before[s, l, g].clone()
    want[:T] *= decay
    assert torch.equal(c.mass[s, l, g], want)
    for name in ("out", "lse", "mass"):
        a, b = getattr(c, name).clone(), getattr(clean, name).clone()
        for x in (a, b):
            (x[s, l, g] if name == "mass" else x[s, :, l, heads]).zero_()
        assert torch.equal(a, b), name
    c.k[s, l, g, :, 5], c.tk[s, :, l, g, 5], c.tv[s, c.tails[s], l, g, 9] = finite
    before = c.mass.clone()
    c.call(decay=decay)
    c.check(decay, before)


def test_a_token_whose_logits_are_minus_infinity_keeps_its_weight():
    """One view token with such a key: its weight only decays, the others' are those of a softmax without it (decay 0.5,
    exact for the token; the others against the plain values of the remaining tokens, in 64 bits)."""
    c = weights_case(lens=(5,), M=2, tails=(3,), seed=72)
    c.q[:, :, :, :, 5] = 0.5
    c.k[:, :, :, 17, 5] = -math.inf
    before = c.mass.clone()
    c.call(decay=0.5)
    torch.cuda.synchronize()
    assert torch.equal(c.mass[:, :, :, 17], 0.5 * before[:, :, :, 17])
    T, r = 5 * c.B, c.H // c.G
    rest = [t for t in range(T) if t != 17]
    for g in range(c.G):
        K = torch.cat([c.k[0, 0, g, rest], c.tk[0, :3 + c.M, 0, g]]).double()
        w = torch.zeros(T - 1, dtype=torch.float64, device="cuda")
        mag = 0.0
        for i in range(c.M):
            Ki = K[:T - 1 + 3 + i + 1]
            q = c.q[0, i, 0, g * r:(g + 1) * r].double()
            w += ((q @ Ki.T) / math.sqrt(128)).softmax(1)[:, :T - 1].sum(0)
            mag = max(mag, ((q.abs() @ Ki.abs().T) / math.sqrt(128)).max().item())
        want = 0.5 * before[0, 0, g, rest].double() + w
        # the bounds of test_gpu_tree.py: a logit is off by 128 * 2^-23 of its terms' magnitudes, twice (its own and the log-sum-exp's)
        tol = w * (2 * 128 * 2.0 ** -23 * mag + 2.0 ** -13 + 2.0 ** -20) + want * 2.0 ** -22
        assert bool(((c.mass[0, 0, g, rest].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_nothing_masked_reaches_the_weights(value):
    """Keys and values behind the view's end and behind the tail, and values of drafted tokens, are not in any weight."""
    kw = dict(ns=2, lens=(3, 5), B=32, M=4, n_q=(4, 2), tails=(9, 2), seed=73)
    c, clean = weights_case(**kw), weights_case(**kw)
    for s in range(2):
        c.k[s, :, :, c.lens[s] * c.B:] = value
        c.v[s, :, :, c.lens[s] * c.B:] = value
        end = c.tails[s] + c.n_q[s]
        c.tk[s, end:] = value
        c.tv[s, end:] = value
        c.tv[s, end - 1, :, :, 7] = value                        # a value that only the last drafted token sees
    c.call(decay=0.5)
    clean.call(decay=0.5)
    torch.cuda.synchronize()
    assert torch.equal(c.mass, clean.mass)
    for s in range(2):
        last = c.n_q[s] - 1
        assert torch.equal(c.lse[s], clean.lse[s]) and torch.equal(c.out[s, :last], clean.out[s, :last])
    c.guards.check()


def test_a_logit_that_is_not_a_number_stays_with_its_head():
    """A NaN among the keys of one KV head makes its rows and the weights of its tokens NaN, as the definition does, and
    touches nothing behind the view's end and no other head."""
    c, clean = weights_case(**RAGGED), weights_case(**RAGGED)
    s, l, g, r = 1, 0, 1, c.H // c.G
    c.k[s, l, g, 130, 3] = math.nan
    c.call(decay=0.5)
    clean.call(decay=0.5)
    torch.cuda.synchronize()
    T = c.lens[s] * c.B
    assert bool(c.mass[s, l, g, :T].isnan().all()) and bool(c.out[s, :, l, g * r:(g + 1) * r].isnan().all())
    assert torch.equal(c.mass[s, l, g, T:], clean.mass[s, l, g, T:])
    c.mass[s, l, g] = clean.mass[s, l, g]
    assert torch.equal(c.mass, clean.mass)
    c.guards.check()


# Which kernel sums the weights: with 296 runs of 2,048 tokens of capacity over all heads (64 heads: 10,240 tokens) or more, up to 4
# rows are one warp's (2,048 tokens a block), up to 8 two warps' (1,024 tokens a block); up to 16 rows, and fewer below those
# capacities, are four warps' (256 tokens a block), more rows eight warps'.  Block sizes of 16 tokens, lengths on either side of
# the blocks' ends, an empty view, a full one, sessions with fewer drafted tokens than the call's.
SUMS = [(M, H, cap) for cap in (640, 639, 645) for M, H in ((1, 32), (2, 32), (3, 8), (5, 8), (1, 8), (7, 8))] + [(3, 32, 640), (8, 40, 640)]


@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("M,H,cap", SUMS)
def test_each_kernel_that_sums_the_weights(M, H, cap, decay):
    lens = (cap, 0, 64, 63, 129, 321, 638, 1)
    c = weights_case(mass_seed=M, ns=8, H=H, G=8, B=16, lens=lens, M=M, n_q=[M, M, M, max(M - 1, 0), M, 1, M, (M + 1) // 2],
                     tails=(0, 5, 130, 0, 1, 64, 17, 2), cap_blocks=cap, seed=300 + M)
    before = c.mass.clone()
    c.call(decay=decay)
    c.check(decay, before)


@pytest.mark.parametrize("unmet", [0, 1, 2])
def test_a_joint_wait_that_runs_out_sets_the_status_word_and_leaves_the_pool_usable(unmet):
    """The MMA thread's wait for three barriers, one of which nobody arrives at: with a limit of 2 ms it gives up, whichever
    of the three it is, reports KVMEM_E_TIMEOUT and returns; a call on the same pool is then right."""
    c = Case(lens=(5,), M=40, seed=80)                           # 160 rows per KV head: two row tiles, all three barriers in use
    assert c.pool.device_status() == 0
    waited = c.pool.selftest_joint_wait_timeout(unmet, 2000)
    assert 2_000_000 <= waited < 500_000_000, f"the wait lasted {waited} ns"
    assert c.pool.device_status() == kvmem.E_TIMEOUT
    assert c.pool.device_status() == 0
    c.call()
    c.check()


def test_the_joint_waits_refusals():
    c = Case(lens=(1,), M=1)
    for unmet, limit_us in ((-1, 1000), (3, 1000), (0, 0), (0, 100001)):
        with pytest.raises(KvmemError) as e:
            c.pool.selftest_joint_wait_timeout(unmet, limit_us)
        assert e.value.status == kvmem.E_INVALID
    assert c.pool.lib.kvmem_selftest_joint_wait_timeout(None, 0, 1000, None, None) == kvmem.E_STATE
    assert c.pool.device_status() == 0


# ---- sizes at the ends of the ranges

@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kw", [
    dict(M=64, H=1024, G=1, lens=(2,), B=32, tails=(9,)),                          # 65,536 rows on one KV head: 256 row groups
    dict(M=1, H=3, G=3, lens=(1,), B=16, tails=(0,), cap_blocks=1, tail_cap=1),   # a capacity below one copy's 64 rows, one tail row
    dict(M=5, H=4, G=2, ns=3, lens=(1, 1, 0), B=16, tails=(11, 0, 3), cap_blocks=1, tail_cap=16),
    dict(M=2, H=2, G=1, lens=(0,), tails=(70001,)),                                # everything in the tail
], ids=["65536 rows", "one row", "one block", "long tail"])
def test_smallest_and_largest(paged, kw):
    c = Case(paged=paged, seed=110, extra=0, **kw)
    c.call()
    c.check()


def test_thousands_of_sessions():
    """4,999 sessions, a few tokens each, some empty; every 97th is compared, and all of them must be written or left."""
    ns = 4999
    c = Case(ns=ns, H=2, G=1, B=16, lens=[(5 * s) % 3 for s in range(ns)], M=2, n_q=[s % 3 for s in range(ns)],
             tails=[(7 * s) % 4 for s in range(ns)], mask="chain", seed=111, cap_blocks=2)
    c.mass = c.guards.empty((ns, 1, 1, c.capb * c.B), torch.float32, fill=0.25)
    c.call(decay=0.5)
    torch.cuda.synchronize()
    live = torch.arange(2).view(1, 2) < c.nq_dev.cpu().view(ns, 1)
    assert torch.equal((c.lse != 55.0).all(3).all(2).cpu(), live)
    for s in range(0, ns, 97):
        one = c.n_q[s]
        if one == 0:
            assert bool((c.mass[s, 0, 0, :c.lens[s] * 16] == 0.125).all())
            continue
        p, T, ref, absv, lse, dx = c.reference(s, 0)
        got = c.out[s, :one, 0].reshape(one * 2, 128).double()
        assert bool(((got - ref).abs() <= (2.0 ** -8 + 2.0 ** -14 + 2 * dx) * absv * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-30).all())
        w = p[:, :T].sum(0)
        want = 0.125 + w
        assert bool(((c.mass[s, 0, 0, :T].double() - want).abs() <= w * (2 * dx + 2.0 ** -13 + 2.0 ** -20) + want * 2.0 ** -22).all())
        assert bool((c.mass[s, 0, 0, T:] == 0.25).all())
    c.guards.check()


@pytest.mark.parametrize("kind", ["heavy", "ties", "zero"])
def test_eviction_by_one_cta_of_more_tokens_than_it_holds(kind):
    """160 heads, a CTA each, two sessions of more than the 36,864 tokens whose weights fit its shared memory; a destination
    whose capacity is no multiple of anything."""
    lens = [580, 0, 3, 601, 1, 0, 2, 9, 5, 1]
    c = EvictCase(ns=10, G=16, B=64, lens=lens, keep=99, sink=5, recent=130, kind=kind, seed=112, dst_cap=99 * 64 + 5)
    c.call()
    c.check()


# ---- the pool's own workspace

def held():
    """Bytes of all live tensors (as asked for, whatever blocks they came out of)."""
    return torch.cuda.memory_stats()["requested_bytes.all.current"]


def own_bytes(c):
    lib, cfg = c.pool.lib, kvmem.C.byref(c.pool.cfg)
    if c.mass is None:
        return lib.kvmem_tree_workspace_bytes(cfg, c.ns, c.M)
    return lib.kvmem_mass_workspace_bytes(cfg, c.ns, c.M, c.capb * c.B)


def three_sizes():
    """Three calls of one pool whose workspaces hold some 83, 157 and 158 MB."""
    cases = [weights_case(lens=(3,), M=16, cap_blocks=blocks, seed=90 + i) for i, blocks in enumerate((2225, 4500, 4525))]
    for c in cases[1:]:
        c.pool = cases[0].pool
    gc.collect()
    return cases


def test_a_workspace_that_grows_gives_the_smaller_one_back():
    cases = three_sizes()
    sizes = [own_bytes(c) for c in cases]
    assert 64 << 20 < sizes[0] < sizes[1] < sizes[2] < 1.02 * sizes[1]
    base = held()
    for c, size in zip(cases, sizes):
        before = c.mass.clone()
        c.call(decay=0.5)
        del before
        assert held() - base == size
    cases[0].call()                                              # a smaller call takes the larger workspace
    assert held() - base == sizes[2]
    cases[0].pool.close()
    assert held() == base
    torch.cuda.synchronize()


@pytest.mark.parametrize("why", ["captured", "captured on its stream", "other stream"])
def test_a_workspace_that_may_still_be_written_is_kept(why):
    """One that a captured graph replays on, or that a call on another stream than its own used, outlives the growth: memory
    handed out afterwards is not written by a replay.  close() gives all of it back."""
    cases = three_sizes()
    sizes = [own_bytes(c) for c in cases]
    small, side, graph = cases[0], torch.cuda.Stream(), None
    torch.cuda.synchronize()
    with torch.cuda.stream(side if why == "captured on its stream" else torch.cuda.current_stream()):
        small.call(decay=0.0)
    torch.cuda.synchronize()
    first = (small.out.clone(), small.lse.clone())
    if why == "other stream":
        with torch.cuda.stream(side):
            small.call(decay=0.0)
    else:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            small.call(decay=0.0)
    torch.cuda.synchronize()
    base = held() - sizes[0]
    cases[1].call(decay=0.0)
    assert held() - base == sizes[0] + sizes[1]
    if graph is not None:
        others = [torch.full((sizes[0],), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
        small.out.zero_()
        small.lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(small.out, first[0]) and torch.equal(small.lse, first[1])
        assert all(bool((o == 0xA5).all()) for o in others)
        del others
    cases[2].call(decay=0.0)                                     # the second was only used on its own stream: given back
    assert held() - base == sizes[0] + sizes[2]
    small.pool.close()
    assert held() - base == 0
    torch.cuda.synchronize()


def test_small_workspaces_that_are_kept_double():
    """Graphs captured at growing sizes: what is kept stays within twice the largest."""
    cases = [Case(lens=(2,), M=M, seed=M) for M in (1, 2, 3, 5, 8, 13, 21, 34, 64)]
    for c in cases[1:]:
        c.pool = cases[0].pool
    gc.collect()
    start, graphs = held(), []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call()
        graphs.append(g)
    assert held() - start <= 4 * own_bytes(cases[-1])      # the newest: at most twice; the ones before: as much
    for c, g in zip(cases, graphs):
        g.replay()
        c.check()


# ---- pools with rotary support

def rotary_pool(c, in_block):
    """c's history in a pool whose pages hold raw keys, or keys rotated by their offset in the block."""
    pool = Pool(c.L, c.H, c.G, 128, c.B, c.ns, c.ns * c.hk.shape[1] // c.B, c.hk.shape[1] // c.B, 0, 2048, 1e6, rope_in_block_keys=in_block)
    for s in range(c.ns):
        pool.append_blocks(s, c.hk[s], c.hv[s])
    return pool


def test_pages_of_raw_keys_are_read_as_they_lie():
    c, plain = (Case(ns=2, L=2, lens=(5, 3), M=6, tails=(9, 70), paged=True, seed=100) for _ in range(2))
    c.pool = rotary_pool(c, False)
    c.call()
    plain.call()
    c.check()
    assert torch.equal(c.out, plain.out) and torch.equal(c.lse, plain.lse)


def test_pages_of_keys_rotated_in_their_block_are_refused():
    """No position makes their angles those of one view: they are materialised first."""
    c = Case(ns=2, lens=(5, 3), M=6, paged=True, seed=101)
    c.pool = rotary_pool(c, True)
    with pytest.raises(KvmemError) as e:
        c.call()
    assert e.value.status == kvmem.E_STATE and "materialize_rope" in str(e.value)
    torch.cuda.synchronize()
    assert bool((c.out == 77.0).all()) and bool((c.lse == 55.0).all())


@pytest.mark.parametrize("in_block", [False, True])
def test_position_consistent_decode_materialises_first(in_block):
    """Drafted tokens at the positions behind a rotated view: the view's keys are those of compact positions, tail and
    queries carry their own, and the result is the attention over them."""
    c = Case(ns=2, L=2, lens=(5, 3), M=6, tails=(9, 70), paged=True, seed=102)
    pool = rotary_pool(c, in_block)
    view = pool.new_view(c.ns, c.capb * c.B)
    pool.materialize_rope(c.sel, c.n_sel, view)
    raw = c.k
    for s in range(c.ns):
        T, end = c.lens[s] * c.B, c.tcap
        pos = torch.arange(T, dtype=torch.int32, device="cuda")
        want = pool.rope_rotate(raw[s, :, :, :T].permute(2, 0, 1, 3).reshape(T, c.L * c.G, 128).contiguous(), pos).view(T, c.L, c.G, 128)
        got = view.k[s, :, :, :T].permute(2, 0, 1, 3).float()
        # in-block keys are rounded once more, 2^-8 of each of the two elements that a rotation mixes, and both results once (2^-8):
        # four times 2^-8 of the head's largest element
        assert bool(((got - want.float()).abs() <= (2.0 ** -7 * want.float().abs().amax(3, keepdim=True) * 2 if in_block else 0.0)).all())
        tpos = torch.arange(T, T + end, dtype=torch.int32, device="cuda")
        c.tk[s] = pool.rope_rotate(c.tk[s].reshape(end, c.L * c.G, 128).contiguous(), tpos).view(end, c.L, c.G, 128)
        qpos = T + c.tails[s] + torch.arange(c.M, dtype=torch.int32, device="cuda")
        c.q[s] = pool.rope_rotate(c.q[s].reshape(c.M, c.L * c.H, 128).contiguous(), qpos).view(c.M, c.L, c.H, 128)
    c.k, c.v, c.pool, c.paged = view.k, view.v, pool, False
    c.call()
    c.check()
