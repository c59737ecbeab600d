"""Attention of drafted tokens over view (or pages) and tail, and the weights it accumulates, against a plain
restatement in 64 bits.

Bounds.  The weights enter the second product rounded once to bf16 (relative 2^-8 at most) and the result is rounded
once to bf16, everything else is fp32: |out - ref| <= 2^-8 sum p|v| + 2^-8 |ref|, plus the fp32 sums, for which 2^-14 sum
p|v| is allowed (a sum of n fp32 terms is off by at most n 2^-24 of the sum of their magnitudes, n <= 1024 here per
accumulation, and 2^-14 covers that with the logits' own error below).  A logit is a sum of 128 exact products: at most
128 * 2^-23 of the sum of their magnitudes (2^-23: tensor-core sums may truncate).  The log-sum-exp inherits the largest
logit error, and a relative error of its sum of at most 2^-24 per term of a running sum (<= 2^12 terms: 2^-12 would be
the very worst; the sums here are split over threads and tiles, so 2^-13 bounds them) with 2^-21 for the exponentials.
A weight has the relative error of its logit and of the log-sum-exp."""
import math

import pytest
import torch

from kvmem_harness import Guards
from paper_2609_04852_b200 import KvmemError, Pool, Tail, View
from paper_2609_04852_b200 import kvmem

pytestmark = pytest.mark.gpu
D = 128


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def random_tree(gen_seed, ns, M, n_q):
    """Ancestor bits, self included; words of padded tokens are garbage on purpose."""
    g = torch.Generator().manual_seed(gen_seed)
    rows = []
    for s in range(ns):
        bits = []
        for i in range(M):
            p = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
            bits.append((1 << i) | (bits[p] if p >= 0 else 0))
        # bits of tokens behind the session's last must not count
        junk = ((1 << 64) - 1) ^ ((1 << n_q[s]) - 1)
        rows.append([b | junk for b in bits])
    return rows


def as_mask(rows):
    return torch.tensor([[b - (1 << 64) if b >= (1 << 63) else b for b in r] for r in rows], dtype=torch.int64, device="cuda")


class Case:
    """One call's inputs and the 64-bit result.  lens: blocks per session in the view (or selected)."""

    def __init__(self, ns=1, L=1, H=8, G=2, B=64, lens=(3,), M=5, n_q=None, tails=None, mask="tree", paged=False, seed=0,
                 cap_blocks=None, tail_cap=None, scale=0.0, extra=2):
        self.ns, self.L, self.H, self.G, self.B, self.M, self.paged, self.scale = ns, L, H, G, B, M, paged, scale
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dev = torch.device("cuda", torch.cuda.current_device())
        self.lens = list(lens)
        self.n_q = [M] * ns if n_q is None else list(n_q)
        self.tails = [7 + s for s in range(ns)] if tails is None else list(tails)
        self.capb = max(max(self.lens), 1) + extra if cap_blocks is None else cap_blocks
        self.tcap = max(self.tails) + M + 3 if tail_cap is None else tail_cap
        T = self.capb * B
        self.q = _normal(gen, ns, M, L, H, D).mul_(1.5).to(torch.bfloat16)
        self.tk, self.tv = (_normal(gen, ns, self.tcap, L, G, D).to(torch.bfloat16) for _ in range(2))
        self.n_sel = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.nq_dev = torch.tensor(self.n_q, dtype=torch.int32, device=dev)
        self.nt_dev = torch.tensor(self.tails, dtype=torch.int32, device=dev)
        if paged:
            hist = self.capb + 5
            perm = torch.randperm(ns * hist + 3, generator=torch.Generator().manual_seed(seed))[:ns * hist].view(ns, hist)
            self.pool = Pool(L, H, G, D, B, ns, ns * hist + 3, hist, dev.index)
            self.hk, self.hv = (_normal(gen, ns, hist * B, L, G, D).to(torch.bfloat16) for _ in range(2))
            for s in range(ns):
                self.pool.append_blocks(s, self.hk[s], self.hv[s], perm[s].tolist())
            self.sel = torch.stack([torch.randperm(hist, generator=torch.Generator().manual_seed(seed + 9 + s))[:self.capb].sort().values
                                    for s in range(ns)]).to(torch.int32).to(dev)
            at = self.sel.long().view(ns, self.capb, 1, 1, 1, 1).expand(ns, self.capb, B, L, G, D)
            self.k, self.v = (x.view(ns, hist, B, L, G, D).gather(1, at).view(ns, T, L, G, D).permute(0, 2, 3, 1, 4)
                              for x in (self.hk, self.hv))
        else:
            self.pool = Pool(L, H, G, D, B, ns, 1, 1, dev.index)
            self.k, self.v = (_normal(gen, ns, L, G, T, D).to(torch.bfloat16) for _ in range(2))
        if isinstance(mask, str):
            self.rows = {"tree": lambda: random_tree(seed, ns, M, self.n_q), "chain": lambda: None,
                         "empty": lambda: [[0] * M for _ in range(ns)],
                         "all": lambda: [[(1 << 64) - 1] * M for _ in range(ns)]}[mask]()
        else:
            self.rows = mask
        self.mask = None if self.rows is None else as_mask(self.rows)
        self.guards = Guards(dev)
        self.out = self.guards.empty((ns, M, L, H, D), torch.bfloat16, fill=77.0)
        self.lse = self.guards.empty((ns, M, L, H), torch.float32, fill=55.0)
        self.mass = None

    def call(self, **kw):
        tail = Tail(self.tk, self.tv, self.nt_dev)
        if self.paged:
            self.pool.paged_tree_attend(self.q, self.sel, self.n_sel, tail, self.out, self.lse, mask=self.mask, n_q=self.nq_dev,
                                        scale=self.scale, **kw)
        elif self.mass is not None:
            self.pool.view_attend_mass(self.q, View(self.k, self.v, self.capb * self.B), self.n_sel, self.mass, self.out, self.lse,
                                       tail=tail, n_q=self.nq_dev, scale=self.scale, **kw)
        else:
            self.pool.view_tree_attend(self.q, View(self.k, self.v, self.capb * self.B), self.n_sel, tail, self.out, self.lse,
                                       mask=self.mask, n_q=self.nq_dev, scale=self.scale, **kw)

    def reference(self, s, lg):
        """(weights [n_q*r][T + tail + drafted], T, out, sum p|v|, lse, logit error bound) of one session and KV head."""
        r, l, g = self.H // self.G, lg // self.G, lg % self.G
        T, nt, nq = min(self.lens[s], self.capb) * self.B, self.tails[s], self.n_q[s]
        K = torch.cat([self.k[s, l, g, :T], self.tk[s, :nt + nq, l, g]]).double()
        V = torch.cat([self.v[s, l, g, :T], self.tv[s, :nt + nq, l, g]]).double()
        q = self.q[s, :nq, l, g * r:(g + 1) * r].reshape(nq * r, D).double()
        sees = torch.ones(nq, T + nt + nq, dtype=torch.bool)
        for i in range(nq):
            bits = (2 << i) - 1 if self.rows is None else self.rows[s][i]
            for j in range(nq):
                sees[i, T + nt + j] = bool((bits >> j) & 1)
        sees = sees.cuda().repeat_interleave(r, 0)
        scale = self.scale or 1.0 / math.sqrt(D)
        x = (q @ K.T) * scale
        x = torch.where(sees, x, torch.full_like(x, -math.inf))
        mag = torch.where(sees, (q.abs() @ K.abs().T) * scale, torch.zeros_like(x))
        top = x.amax(1, keepdim=True) if x.shape[1] else torch.full((x.shape[0], 1), -math.inf, dtype=torch.float64, device="cuda")
        e = torch.where(sees, (x - torch.where(top > -math.inf, top, torch.zeros_like(top))).exp(), torch.zeros_like(x))
        z = e.sum(1, keepdim=True)
        p = e / torch.where(z > 0, z, torch.ones_like(z))
        out, absv = torch.zeros_like(q), torch.zeros_like(q)
        # a token counts only where it is seen: 0 * NaN must not get in
        seen_any = sees.any(0)
        p_, V_ = p[:, seen_any], V[seen_any]
        out, absv = p_ @ V_, p_ @ V_.abs()
        lse = torch.where(z > 0, top + z.log(), torch.full_like(z, -math.inf)).squeeze(1)
        return p, T, out, absv, lse, 128 * 2.0 ** -23 * (mag.max().item() if mag.numel() else 0.0)

    def check(self, decay=None, mass0=None):
        torch.cuda.synchronize()
        assert self.pool.device_status() == 0
        r = self.H // self.G
        for s in range(self.ns):
            nq = self.n_q[s]
            assert bool((self.out[s, nq:] == 77.0).all()) and bool((self.lse[s, nq:] == 55.0).all()), "padded tokens were written"
            for lg in range(self.L * self.G):
                l, g = lg // self.G, lg % self.G
                p, T, ref, absv, lse, dx = self.reference(s, lg)
                got = self.out[s, :nq, l, g * r:(g + 1) * r].reshape(nq * r, D).double()
                tol = (2.0 ** -8 + 2.0 ** -14 + 2 * dx) * absv * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-30
                bad = (got - ref).abs() > tol
                assert not bool(bad.any()), (s, lg, ((got - ref).abs() / tol).max().item())
                gl = self.lse[s, :nq, l, g * r:(g + 1) * r].reshape(-1).double()
                ltol = dx + 2.0 ** -13 + 2.0 ** -21 + 2.0 ** -22 * lse.abs().nan_to_num(0, 0, 0)
                fine = lse > -math.inf
                assert bool((gl[~fine] == -math.inf).all())
                assert bool(((gl - lse).abs() <= ltol)[fine].all()), (s, lg, (gl - lse).abs()[fine].max().item())
                if self.mass is not None:
                    w = p[:, :T].sum(0)
                    m0 = mass0[s, l, g].double()
                    gm = self.mass[s, l, g].double()
                    assert bool((gm[T:] == m0[T:]).all()), "weights behind the view's end were written"
                    want = decay * m0[:T] + w
                    mt = w * (2 * dx + 2.0 ** -13 + 2.0 ** -20) + want.abs() * 2.0 ** -22 + 1e-37
                    assert bool(((gm[:T] - want).abs() <= mt).all()), (s, lg, ((gm[:T] - want).abs() / mt).max().item())
        self.guards.check()


GEOMETRIES = [
    dict(),                                                            # 8 heads over 2, five drafted
    dict(M=1, tails=(0,), mask="chain"),                               # a single token and no tail
    dict(M=1, H=1, G=1, lens=(1,), tails=(0,)),                        # one row in all
    dict(M=64, H=16, G=2, lens=(5,)),                                  # 512 rows per KV head
    dict(M=33, H=8, G=8, lens=(4,), tails=(100,)),                     # no head sharing, odd tree
    dict(M=17, H=10, G=2, lens=(9,), B=16, tails=(1,)),                # five heads on a KV head, 16-token blocks
    dict(M=26, H=20, G=4, lens=(2,), B=32),                            # 130 rows: two rows past a tile of 128
    dict(M=32, H=8, G=2, lens=(7,)),                                   # exactly 128 rows
    dict(M=64, H=8, G=2, lens=(7,), tails=(200,)),                     # exactly 256 rows, a tail of several tiles
    dict(ns=3, L=2, lens=(3, 0, 11), M=6, n_q=(6, 1, 4), tails=(5, 0, 130), B=32),     # ragged batch, one empty view
    dict(ns=4, lens=(1, 40, 2, 0), M=9, n_q=(0, 9, 3, 2), tails=(3, 64, 0, 0), B=16),  # a session without a token
    dict(ns=2, lens=(0, 0), tails=(0, 0), M=4),                        # drafted tokens alone
    dict(ns=2, lens=(20, 3), M=12, B=128, tails=(61, 127)),
    dict(lens=(6,), M=4, B=64, tails=(300,), mask="all"),
    dict(lens=(30,), M=8, B=64, scale=0.02),
    dict(M=64, H=64, G=1, lens=(2,)),                                  # 4,096 rows on one KV head: sixteen row groups
    dict(M=1, H=128, G=1, lens=(9,), mask="chain"),                    # a single token, 128 heads on a KV head
]


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("i", range(len(GEOMETRIES)))
def test_tree_attention_matches_the_definition(i, paged):
    c = Case(paged=paged, seed=10 * i + paged, **GEOMETRIES[i])
    c.call()
    c.check()


# Many tiles per CTA, segments that begin and end anywhere, ragged ends behind full tiles: (the ring of tiles has wrapped
# around several times when a masked tile comes up)
LONG = [
    dict(ns=4, L=2, H=16, G=4, lens=(300, 77, 129, 255), M=12, n_q=(12, 5, 9, 1), tails=(90, 3, 40, 200)),     # 48 rows per KV head
    dict(ns=3, H=32, G=8, lens=(501, 33, 250), M=16, B=32, tails=(50, 129, 0)),                                   # 64 rows
    dict(ns=3, H=16, G=2, lens=(400, 1, 222), M=31, n_q=(31, 31, 10), B=48, tails=(700, 5, 64)),               # 248 and 80 rows
    dict(ns=2, H=16, G=2, lens=(300, 299), M=33, n_q=(33, 32), tails=(600, 100), mask="all"),                  # 264 and 256 rows
    dict(ns=8, H=32, G=8, lens=(200, 52, 73, 95, 116, 137, 158, 0), M=4, tails=(33, 3, 7, 11, 14, 18, 22, 29), mask="chain"),
    dict(ns=1, H=4, G=1, lens=(3001,), M=7, B=16, tails=(1000,)),                                                 # one head on all SMs
    dict(ns=4, H=16, G=2, lens=(100, 3, 57, 9), M=48, n_q=(48, 17, 16, 0), tails=(500, 0, 30, 4)),                # 384, 136, 128, 0 rows
    dict(ns=2, H=16, G=2, lens=(0, 1), M=64, n_q=(64, 33), tails=(0, 70)),                                       # 512 and 264, few tiles
]


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_long_and_ragged_views(i, paged):
    if paged and LONG[i].get("B", 64) == 48:
        pytest.skip("a block size the pages do not take")
    c = Case(paged=paged, seed=200 + i, **LONG[i])
    for _ in range(3):
        c.out.fill_(77.0); c.lse.fill_(55.0)
        c.call()
        c.check()


@pytest.mark.parametrize("mass", [False, True])
def test_many_sessions(mass):
    """More sessions than a warp has lanes, most of them short, some empty, some without a drafted token."""
    ns = 101
    c = Case(ns=ns, H=8, G=2, B=16, lens=[(7 * s) % 23 if s % 5 else 0 for s in range(ns)], M=3, n_q=[s % 4 for s in range(ns)],
             tails=[(11 * s) % 41 for s in range(ns)], mask="chain" if mass else "tree", seed=9, cap_blocks=23)
    before = None
    if mass:
        c.mass = c.guards.empty((ns, 1, 2, c.capb * c.B), torch.float32, fill=0.25)
        before = c.mass.clone()
    c.call(**({"decay": 0.5} if mass else {}))
    c.check(0.5, before)


def test_the_same_bits_from_run_to_run():
    c = Case(seed=3, **LONG[0])
    c.call()
    first = (c.out.clone(), c.lse.clone())
    for _ in range(10):
        c.call()
    assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


@pytest.mark.parametrize("i", [1, 4])
def test_weights_over_long_and_ragged_views(i):
    c = Case(seed=230 + i, **{**LONG[i], "mask": "chain", "M": 4})
    c.mass = c.guards.empty((c.ns, c.L, c.G, c.capb * c.B), torch.float32)
    c.call(decay=0.5)
    c.check(0.5, torch.zeros_like(c.mass))


@pytest.mark.parametrize("B,lens", [(48, (5,)), (80, (3,)), (240, (2,)), (256, (2,)), (192, (3,)), (112, (1,))])
def test_block_sizes_of_the_view(B, lens):
    c = Case(B=B, lens=lens, seed=B)
    c.call()
    c.check()


@pytest.mark.parametrize("B,lens", [(256, (2,)), (192, (3,))])
def test_block_sizes_of_the_pages(B, lens):
    c = Case(B=B, lens=lens, seed=B, paged=True)
    c.call()
    c.check()


@pytest.mark.parametrize("paged", [False, True])
def test_a_token_that_sees_nothing(paged):
    """Empty view, no committed tail and an empty mask word: out = 0 and lse = -inf; its neighbours are ordinary."""
    rows = [[0, 0b10, 0b110, 0, 0b10000], [0b1, 0, 0b100, 0b1000, 0]]
    c = Case(ns=2, lens=(0, 0), tails=(0, 0), M=5, mask=rows, paged=paged)
    c.call()
    c.check()
    assert bool((c.out[0, 0] == 0).all()) and bool((c.lse[0, 3] == -math.inf).all())


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_nothing_reaches_a_result_that_is_masked(paged, value):
    """Whatever the memory behind the view's end, behind the tail and in drafted tokens of other branches holds."""
    M = 6
    rows = [[1 << i | 1 for i in range(M)] for _ in range(2)]        # every token sees token 0 and itself
    c = Case(ns=2, lens=(3, 5), B=32, M=M, n_q=(6, 4), tails=(9, 2), mask=rows, paged=paged, seed=3)
    if not paged:
        for s in range(2):
            c.k[s, :, :, c.lens[s] * c.B:] = value
            c.v[s, :, :, c.lens[s] * c.B:] = value
    for s in range(2):
        end = c.tails[s] + c.n_q[s]
        c.tk[s, end:] = value
        c.tv[s, end:] = value
    # token 3 holds the value: its own rows turn into what arithmetic makes of it, all the others stay clean
    c.tk[:, torch.tensor([c.tails[0] + 3]).cuda(), :, :, 5] = value
    clean = Case(ns=2, lens=(3, 5), B=32, M=M, n_q=(6, 4), tails=(9, 2), mask=rows, paged=paged, seed=3)
    c.tv[0, c.tails[0] + 3, :, :, 7] = value
    c.call()
    clean.call()
    torch.cuda.synchronize()
    for i in (0, 1, 2, 4, 5):
        assert torch.equal(c.out[0, i], clean.out[0, i]) and torch.equal(c.lse[0, i], clean.lse[0, i]), i
    c.guards.check()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_a_visible_value_that_is_not_finite_reaches_the_tokens_that_see_it(value):
    M = 4
    rows = [[0b0001, 0b0011, 0b0101, 0b1001]]
    c = Case(lens=(3,), M=M, mask=rows, seed=5)
    clean = Case(lens=(3,), M=M, mask=rows, seed=5)
    c.tv[0, c.tails[0] + 1, :, :, 9] = value
    c.call()
    clean.call()
    torch.cuda.synchronize()
    for i in range(M):
        same = torch.ones(D, dtype=torch.bool)
        if i == 1:
            same[9] = False
            got = c.out[0, i, :, :, 9].float()
            assert bool(got.isnan().all() if math.isnan(value) else (got == value).all())
        assert torch.equal(c.out[0, i][..., same.cuda()], clean.out[0, i][..., same.cuda()])
        assert torch.equal(c.lse[0, i], clean.lse[0, i])


def test_large_logits_and_growing_maxima():
    """Keys that grow along the view, so that the running maximum moves in every tile; logits up to about 200."""
    c = Case(lens=(24,), M=7, seed=8, scale=0.5)
    ramp = torch.linspace(0.1, 4.0, c.k.shape[3], device="cuda").view(1, 1, 1, -1, 1)
    c.k = (c.k.float() * ramp).to(torch.bfloat16)
    c.call()
    c.check()


def test_without_a_tail_the_view_alone_counts():
    c = Case(lens=(5,), M=3, tails=(0,), mask="chain")
    view = View(c.k, c.v, c.capb * c.B)
    c.pool.view_tree_attend(c.q, view, c.n_sel, None, c.out, c.lse)
    ref_out, ref_lse = c.pool.new_outputs(1, 3)
    c.pool.view_attend(c.q, view, c.n_sel, ref_out, ref_lse)
    torch.cuda.synchronize()
    # the two attention kernels round the weights alike (2^-8 each) and this one its result (2^-8)
    assert bool(((c.lse - ref_lse).abs() <= 1e-4).all())
    c2 = Case(lens=(5,), M=3, tails=(0,), mask="empty")
    c2.call()
    c2.check()
    assert bool(((c.out.float() - c2.out.float()).abs() <= 2.0 ** -7 * c2.out.float().abs() + 1e-6).all())


@pytest.mark.parametrize("bad", [-3, 1 << 20])
def test_a_tail_length_out_of_range_is_clamped_and_reported(bad):
    c = Case(lens=(2,), M=3, tails=(4,), tail_cap=9, mask="chain")
    c.nt_dev.fill_(bad)
    c.call()
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE
    c.tails = [0 if bad < 0 else 6]
    c.check()


def test_counts_out_of_range_are_clamped():
    c = Case(ns=2, lens=(2, 2), M=3, n_q=(3, 0), cap_blocks=2, extra=0)
    c.n_sel[0], c.n_sel[1] = 1 << 30, -5
    c.nq_dev[0], c.nq_dev[1] = 1000, -7
    c.lens = [2, 0]
    c.call()
    c.check()


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_an_id_out_of_range_is_reported(bad):
    c = Case(lens=(4,), M=3, paged=True)
    c.sel[0, 2] = bad
    c.call()
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE
    c.guards.check()


def test_ids_may_repeat_and_come_in_any_order():
    """The selected blocks are read in the order of sel_ids; a block that is named twice counts twice."""
    c = Case(ns=2, lens=(7, 5), B=32, M=4, paged=True, seed=14)
    c.sel[0, :7] = torch.tensor([6, 0, 6, 3, 1, 0, 6], dtype=torch.int32)
    c.sel[1, :5] = torch.tensor([4, 4, 4, 4, 2], dtype=torch.int32)
    hist = c.hk.shape[1] // c.B
    at = c.sel.long().clamp(max=hist - 1).view(2, c.capb, 1, 1, 1, 1).expand(2, c.capb, c.B, c.L, c.G, D)
    c.k, c.v = (x.view(2, hist, c.B, c.L, c.G, D).gather(1, at).view(2, c.capb * c.B, c.L, c.G, D).permute(0, 2, 3, 1, 4)
                for x in (c.hk, c.hv))
    c.call()
    c.check()


def test_some_of_a_pools_sessions():
    c = Case(ns=4, lens=(3, 9, 0, 6), M=5, paged=True, seed=15, n_q=(5, 2, 4, 5))
    whole_out, whole_lse = torch.full_like(c.out, 77.0), torch.full_like(c.lse, 55.0)
    c.call()
    whole_out.copy_(c.out); whole_lse.copy_(c.lse)
    part = slice(1, 3)
    out, lse = torch.full_like(c.out[part].contiguous(), 77.0), torch.full_like(c.lse[part].contiguous(), 55.0)
    c.pool.paged_tree_attend(c.q[part].contiguous(), c.sel[part].contiguous(), c.n_sel[part].contiguous(),
                             Tail(c.tk[part].contiguous(), c.tv[part].contiguous(), c.nt_dev[part].contiguous()), out, lse,
                             mask=c.mask[part].contiguous(), n_q=c.nq_dev[part].contiguous(), session_first=1)
    torch.cuda.synchronize()
    # other cuts of the line, other roundings of the same sums: within the roundings of the weights and the result
    assert bool(((out.float() - whole_out[part].float()).abs() <= 2.0 ** -6 * whole_out[part].float().abs() + 1e-3).all())
    assert bool(((lse - whole_lse[part]).abs() <= 1e-4)[lse > -math.inf].all())


def test_with_plain_launches():
    from paper_2609_04852_b200 import set_option
    c = Case(seed=16, **LONG[0])
    c.call()
    torch.cuda.synchronize()
    first = c.out.clone()
    set_option("pdl", 0)
    try:
        c.out.fill_(77.0); c.lse.fill_(55.0)
        c.call()
        c.check()
    finally:
        set_option("pdl", 1)
    assert torch.equal(c.out, first)


def test_a_first_call_may_be_captured():
    """A process whose first calls are captured: nothing they need is set up by an eager call before."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2609_04852_b200 import Pool, Tail, View
pool = Pool(1, 8, 2, 128, 64, 1, 1, 1, 0)
g = torch.Generator(device="cuda").manual_seed(1)
rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
def buffers(M):
    return rnd(1, M, 1, 8, 128), torch.zeros(1, M, 1, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, M, 1, 8, device="cuda")
view, n = View(rnd(1, 1, 2, 640, 128), rnd(1, 1, 2, 640, 128), 640), torch.tensor([9], dtype=torch.int32, device="cuda")
tail = Tail(rnd(1, 80, 1, 2, 128), rnd(1, 80, 1, 2, 128), torch.tensor([5], dtype=torch.int32, device="cuda"))
mass, dm = torch.zeros(1, 1, 2, 640, device="cuda"), torch.zeros(1, 1, 2, 256, device="cuda")
dst, nd = View(torch.zeros(1, 1, 2, 256, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 2, 256, 128, dtype=torch.bfloat16, device="cuda"), 256), torch.zeros(1, dtype=torch.int32, device="cuda")
few, many, one = buffers(3), buffers(64), buffers(1)
def all_calls():
    pool.view_tree_attend(few[0], view, n, tail, few[1], few[2])
    pool.view_tree_attend(many[0], view, n, tail, many[1], many[2])
    pool.view_attend_mass(one[0], view, n, mass, one[1], one[2], tail=tail, decay=0.0)
    pool.view_evict(view, n, mass, dst, nd, dm, n_sink_tokens=3)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    all_calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (few[1], many[1], one[1], mass, dst.k, dm, nd)]
assert pool.device_status() == 0 and nd.item() == 4 and float(mass.sum()) > 0 and all(float(t.float().abs().sum()) > 0 for t in got)
all_calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (few[1], many[1], one[1], mass, dst.k, dm, nd)))
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]


MASS = [
    dict(M=1, tails=(0,), lens=(3,)),
    dict(M=1, lens=(40,), H=32, G=8),
    dict(M=4, lens=(9,), B=32, L=2),
    dict(M=16, H=8, G=2, lens=(5,)),                                   # 64 rows per KV head
    dict(M=13, H=5, G=1, lens=(70,), B=16, tails=(150,)),              # 65 rows would be one too many: 13 * 5 = 65
    dict(ns=3, M=3, n_q=(3, 1, 0), lens=(0, 7, 2), tails=(2, 0, 5)),
]


@pytest.mark.parametrize("decay", [1.0, 0.0, 0.5])
@pytest.mark.parametrize("i", range(len(MASS)))
def test_accumulated_weights(i, decay):
    spec = dict(MASS[i])
    if spec["M"] * spec.get("H", 8) // spec.get("G", 2) > 64:
        spec["M"] = 12
    c = Case(seed=40 + i, mask="chain", **spec)
    c.mass = c.guards.empty((c.ns, c.L, c.G, c.capb * c.B), torch.float32)
    c.mass.copy_(torch.rand(c.mass.shape, generator=torch.Generator().manual_seed(i)))
    before = c.mass.clone()
    c.call(decay=decay)
    c.check(decay, before)
    # the weights of a step add up to its query rows, less what the tail took
    if decay == 0.0 and max(c.tails) == 0 and c.M == 1:
        T = c.lens[0] * c.B
        drafted = c.reference(0, 0)[0][:, T:].sum().item()
        assert abs(c.mass[0, 0, 0, :T].double().sum().item() + drafted - c.H // c.G) < 1e-3


def test_weights_over_several_steps_are_the_same_bits_again():
    res = []
    for _ in range(2):
        c = Case(M=2, lens=(20,), mask="chain", seed=77)
        c.mass = torch.zeros(1, 1, 2, c.capb * c.B, device="cuda")
        for _ in range(5):
            c.call(decay=0.9)
        torch.cuda.synchronize()
        res.append((c.mass.clone(), c.out.clone(), c.lse.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("mass", [False, True])
def test_captured_calls_follow_lengths_on_the_device(mass):
    """One captured call, replayed after lengths, tokens and masks changed on the device."""
    c = Case(ns=2, lens=(4, 2), M=4, n_q=(4, 3), mask="chain" if mass else "tree", tails=(3, 8), seed=21)
    if mass:
        c.mass = torch.zeros(c.ns, c.L, c.G, c.capb * c.B, device="cuda")
    c.call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call(**({"decay": 0.0} if mass else {}))
    for lens, nq, tails in (((6, 1), (2, 4), (0, 5)), ((0, 4), (4, 1), (9, 9))):
        c.lens, c.n_q, c.tails = list(lens), list(nq), list(tails)
        c.n_sel.copy_(torch.tensor(lens)); c.nq_dev.copy_(torch.tensor(nq)); c.nt_dev.copy_(torch.tensor(tails))
        c.tk.copy_(c.tk.flip(1))
        c.out.fill_(77.0); c.lse.fill_(55.0)
        if not mass:
            c.rows = random_tree(sum(lens), c.ns, c.M, c.n_q)
            c.mask.copy_(as_mask(c.rows))
        before = None if not mass else c.mass.clone()
        g.replay()
        c.check(0.0, before)


def test_two_streams_with_their_own_workspaces():
    cases = [Case(ns=2, lens=(30, 12), M=8, seed=60 + i) for i in range(2)]
    need = [c.pool.lib.kvmem_tree_workspace_bytes(kvmem.C.byref(c.pool.cfg), c.ns, c.M) for c in cases]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in need]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, w, st in zip(cases, ws, streams):
            with torch.cuda.stream(st):
                c.call(workspace=w)
    for c in cases:
        c.check()


def test_offsets_past_32_bits():
    """A view of more than 2^32 bytes and 2^31 elements: the last session's rows lie behind both."""
    ns, G, cap = 9, 8, 262144
    dev = torch.device("cuda", 0)
    pool = Pool(1, 32, G, D, 64, ns, 1, 1, 0)
    k = torch.zeros(ns, 1, G, cap, D, dtype=torch.bfloat16, device=dev)
    v = torch.zeros_like(k)
    c = Case(ns=1, H=32, G=G, lens=(90,), M=3, seed=31, mask="chain")
    T = 90 * 64
    k[ns - 1, :, :, :T], v[ns - 1, :, :, :T] = c.k[0, :, :, :T], c.v[0, :, :, :T]
    lens = torch.zeros(ns, dtype=torch.int32, device=dev)
    lens[ns - 1] = 90
    exp = lambda x: torch.cat([torch.zeros(ns - 1, *x.shape[1:], dtype=x.dtype, device=dev), x])   # noqa: E731
    out, lse = torch.zeros(ns, 3, 1, 32, D, dtype=torch.bfloat16, device=dev), torch.zeros(ns, 3, 1, 32, device=dev)
    mass = torch.zeros(ns, 1, G, cap, device=dev)
    tail = Tail(exp(c.tk), exp(c.tv), exp(c.nt_dev))
    pool.view_attend_mass(exp(c.q), View(k, v, cap), lens, mass, out, lse, tail=tail)
    torch.cuda.synchronize()
    c.mass = torch.zeros(1, 1, G, c.capb * 64, device=dev)
    c.out.copy_(out[ns - 1:]); c.lse.copy_(lse[ns - 1:]); c.mass.copy_(mass[ns - 1:, :, :, :c.capb * 64])
    c.check(1.0, torch.zeros_like(c.mass))
    assert bool((mass[:ns - 1] == 0).all()) and bool((mass[ns - 1, :, :, T:] == 0).all())


def test_refusals():
    c = Case(lens=(2,), M=3, mask="tree")
    view, tail = View(c.k, c.v, c.capb * c.B), Tail(c.tk, c.tv, c.nt_dev)

    def raises(kind, status=None, q=c.q, view=view, n_sel=c.n_sel, tail=tail, out=c.out, lse=c.lse, **kw):
        with pytest.raises(kind) as e:
            c.pool.view_tree_attend(q, view, n_sel, tail, out, lse, **kw)
        if status is not None:
            assert e.value.status == status

    raises(ValueError, q=c.q.float())
    raises(ValueError, q=c.q[0])
    raises(ValueError, q=c.q.transpose(1, 2))
    raises(ValueError, out=c.out.float())
    raises(ValueError, lse=c.lse[:, :2])
    raises(ValueError, n_sel=c.n_sel.long())
    raises(ValueError, n_sel=c.n_sel.cpu())
    raises(ValueError, mask=c.mask[:, :2])
    raises(ValueError, mask=c.mask.int())
    raises(ValueError, tail=Tail(c.tk[:, :, :, :1], c.tv, c.nt_dev))
    raises(ValueError, view=View(c.k, c.v, c.capb * c.B - 64))
    raises(KvmemError, kvmem.E_INVALID, tail=Tail(c.tk[:, :2].contiguous(), c.tv[:, :2].contiguous(), c.nt_dev))
    raises(KvmemError, kvmem.E_INVALID, tail=None, mask=c.mask)
    raises(KvmemError, kvmem.E_INVALID, scale=-1.0)
    raises(KvmemError, kvmem.E_INVALID, scale=math.nan)
    raises(KvmemError, kvmem.E_CAPACITY, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    wide = torch.zeros(1, 65, 1, 8, D, dtype=torch.bfloat16, device="cuda")
    raises(KvmemError, kvmem.E_INVALID, q=wide, out=torch.zeros_like(wide), lse=torch.zeros(1, 65, 1, 8, device="cuda"))
    # weights: at most 64 query rows per KV head, a decay that is a number
    m = Case(lens=(2,), M=17, mask="chain")
    mass = torch.zeros(1, 1, 2, m.capb * m.B, device="cuda")
    mv, mt = View(m.k, m.v, m.capb * m.B), Tail(m.tk, m.tv, m.nt_dev)
    with pytest.raises(KvmemError) as e:
        m.pool.view_attend_mass(m.q, mv, m.n_sel, mass, m.out, m.lse, tail=mt)
    assert e.value.status == kvmem.E_UNSUPPORTED
    for decay in (-0.5, math.inf, math.nan):
        with pytest.raises(KvmemError) as e:
            c.pool.view_attend_mass(c.q, view, c.n_sel, mass[:, :, :, :c.capb * c.B].contiguous(), c.out, c.lse, tail=tail, decay=decay)
        assert e.value.status == kvmem.E_INVALID
    with pytest.raises(ValueError):
        c.pool.view_attend_mass(c.q, view, c.n_sel, mass[:, :, :1], c.out, c.lse, tail=tail)
    torch.cuda.synchronize()
    assert bool((c.out == 77.0).all()), "a refused call wrote"
    # pages the bf16 kernels cannot read, a block size the paged form does not take
    p8 = Pool(1, 8, 2, D, 64, 1, 4, 4, 0, fp8_pages=True)
    sel = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    for pool, status in ((p8, kvmem.E_STATE), (Pool(1, 8, 2, D, 48, 1, 4, 4, 0), kvmem.E_UNSUPPORTED),
                         (Pool(1, 8, 2, 64, 64, 1, 4, 4, 0), None)):
        if status is None:                       # head_dim 64: every shape follows the pool's
            q = torch.zeros(1, 3, 1, 8, 64, dtype=torch.bfloat16, device="cuda")
            tl = Tail(torch.zeros(1, 9, 1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 9, 1, 2, 64, dtype=torch.bfloat16, device="cuda"), c.nt_dev)
            with pytest.raises(KvmemError) as e:
                pool.paged_tree_attend(q, sel, c.n_sel, tl, torch.zeros_like(q), torch.zeros(1, 3, 1, 8, device="cuda"))
            assert e.value.status == kvmem.E_UNSUPPORTED
            continue
        with pytest.raises(KvmemError) as e:
            pool.paged_tree_attend(c.q, sel, c.n_sel, tail, c.out, c.lse, mask=c.mask)
        assert e.value.status == status
    with pytest.raises(KvmemError) as e:
        Case(lens=(2,), M=3, paged=True).pool.paged_tree_attend(c.q, sel, c.n_sel, tail, c.out, c.lse, mask=c.mask, session_first=1)
    assert e.value.status == kvmem.E_INVALID
