"""Attention of a prompt chunk over view and tail against a plain restatement in 64 bits.

Bounds.  The weights enter the second product rounded once to bf16 (relative 2^-8 at most), the result is rounded once to bf16,
everything else is fp32: |out - ref| <= 2^-8 sum p|v| + 2^-8 |ref|, plus fp32 sums over n tokens, n 2^-23 of the sum of their
magnitudes (2^-23: tensor-core sums may truncate), in the numerator and in the denominator, and what a logit's own error dx does to
a weight on either side of the fraction, 2 dx.  A logit is a sum of 128 exact products: dx = 128 * 2^-23 of the sum of their
magnitudes, which also covers its scaling (three roundings of 2^-24).  The log-sum-exp inherits dx, a relative error of n 2^-24 of its
sum, 2^-21 for the exponentials, and two roundings of its own."""
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


class Chunk:
    """One call's inputs and the 64-bit result.  lens: blocks of each session in the view; tails None: no tail."""

    def __init__(self, ns=1, L=1, H=8, G=2, B=64, lens=(3,), M=100, n_q=None, tails=(7,), seed=0, extra=2, scale=0.0, tail_extra=3):
        self.ns, self.L, self.H, self.G, self.B, self.M, self.scale = ns, L, H, G, B, M, scale
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dev = torch.device("cuda", torch.cuda.current_device())
        self.lens = list(lens)
        self.n_q = [M] * ns if n_q is None else list(n_q)
        self.has_tail = tails is not None
        self.tails = [0] * ns if tails is None else [tails[s % len(tails)] for s in range(ns)]
        self.capb = max(max(self.lens), 1) + extra
        T = self.capb * B
        self.q = _normal(gen, ns, M, L, H, D).mul_(1.5).to(torch.bfloat16)
        self.k, self.v = (_normal(gen, ns, L, G, T, D).to(torch.bfloat16) for _ in range(2))
        self.tcap = max(self.tails) + M + tail_extra
        self.tk, self.tv = (_normal(gen, ns, self.tcap, L, G, D).to(torch.bfloat16) for _ in range(2))
        self.n_sel, self.nq_dev, self.nt_dev = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (self.lens, self.n_q, self.tails))
        self.pool = Pool(L, H, G, D, B, ns, 1, 1, dev.index)
        self.guards = Guards(dev)
        self.out = self.guards.empty((ns, M, L, H, D), torch.bfloat16, fill=77.0)
        self.lse = self.guards.empty((ns, M, L, H), torch.float32, fill=55.0)

    def call(self, **kw):
        tail = Tail(self.tk, self.tv, self.nt_dev) if self.has_tail else None
        self.pool.view_prefill_attend(self.q, View(self.k, self.v, self.capb * self.B), self.n_sel, tail, self.out, self.lse,
                                      n_q=self.nq_dev, scale=self.scale, **kw)

    def reference(self, s, l, h):
        """(out, sum p|v|, lse, logit error bound, tokens) of one session's query head."""
        g = h // (self.H // self.G)
        T, nt, nq = min(self.lens[s], self.capb) * self.B, self.tails[s], self.n_q[s]
        K, V = self.k[s, l, g, :T], self.v[s, l, g, :T]
        if self.has_tail:
            K, V = torch.cat([K, self.tk[s, :nt + nq, l, g]]), torch.cat([V, self.tv[s, :nt + nq, l, g]])
        K, V, q = K.double(), V.double(), self.q[s, :nq, l, h].double()
        n = K.shape[0]
        i = torch.arange(nq, device="cuda").view(-1, 1)
        sees = torch.arange(n, device="cuda").view(1, -1) <= (T + nt + i if self.has_tail else T - 1 + 0 * i)
        scale = self.scale or 1.0 / math.sqrt(D)
        x = torch.where(sees, (q @ K.T) * scale, -math.inf)
        dx = 128 * 2.0 ** -23 * float(((q.abs() @ K.abs().T) * scale).max()) if n and nq else 0.0
        lse = torch.logsumexp(x, 1) if n else torch.full((nq,), -math.inf, dtype=torch.float64, device="cuda")
        p = torch.where(sees & (lse > -math.inf).view(-1, 1), (x - lse.view(-1, 1)).exp(), 0.0)
        return p @ V, p @ V.abs(), lse, dx, n

    def check(self, status=0):
        torch.cuda.synchronize()
        assert self.pool.device_status() == status
        for s in range(self.ns):
            nq = self.n_q[s]
            assert bool((self.out[s, nq:] == 77.0).all()) and bool((self.lse[s, nq:] == 55.0).all()), "padded tokens were written"
            for l in range(self.L):
                for h in range(self.H):
                    ref, absv, lse, dx, n = self.reference(s, l, h)
                    got, gl = self.out[s, :nq, l, h].double(), self.lse[s, :nq, l, h].double()
                    tol = (2.0 ** -8 + 2 * n * 2.0 ** -23 + 2 * dx) * absv * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-30
                    assert bool(((got - ref).abs() <= tol).all()), (s, l, h, ((got - ref).abs() / tol).max().item())
                    fine = lse > -math.inf
                    ltol = dx + n * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -22 * lse[fine].abs()
                    assert bool((gl[~fine] == -math.inf).all())
                    assert bool(((gl - lse).abs()[fine] <= ltol).all()), (s, l, h, (gl - lse).abs()[fine].max().item())
        self.guards.check()


GEOMETRIES = [
    dict(M=1, tails=(0,)),                                             # a single token
    dict(M=2, H=1, G=1, lens=(1,), tails=(0,)),                        # two rows in all
    dict(M=65),                                                        # one more than a mask word holds
    dict(M=100, tails=None),                                           # the view alone
    dict(M=100, lens=(0,), tails=(0,)),                                # the chunk alone
    dict(M=9, lens=(0,), tails=None),                                  # nothing to see: out = 0, lse = -inf
    dict(M=128, H=2, G=2, lens=(2,), tails=(0,)),                      # one full row tile of 128 tokens, no head sharing
    dict(M=129, H=2, G=2, lens=(2,), tails=(1,)),                      # one row in the second
    dict(M=256, H=2, G=2, lens=(2,), tails=(128,)),                    # exactly a group, tails that end with a tile
    dict(M=257, H=2, G=2, lens=(2,), tails=(127,)),
    dict(M=333, H=10, G=2, B=16, lens=(9,), tails=(1,)),               # five heads on a KV head, 16-token blocks: 125 rows of 128
    dict(M=70, H=21, G=3, B=48, lens=(4,), tails=(60,)),               # seven heads on a KV head
    dict(M=5, H=128, G=1, lens=(2,), tails=(3,)),                      # 128 heads on a KV head, few tokens
    dict(M=70, H=128, G=1, lens=(2,), tails=(3,)),                     # a token fills a row tile
    dict(M=67, H=71, G=1, lens=(2,), tails=(3,)),                      # 71: a token a row tile, 57 rows idle
    dict(M=66, H=3, G=3, lens=(1,), tails=(0,)),                       # one item a head, half of it idle
    dict(M=66, lens=(0,), tails=None),                                 # nothing to see, in a long chunk
    dict(ns=3, M=100, lens=(0, 2, 0), n_q=(100, 3, 100), tails=None),  # nothing or a view
    dict(M=90, H=66, G=2, lens=(1,), tails=(0,)),                      # 33: three tokens a row tile
    dict(ns=3, L=2, M=150, lens=(3, 0, 11), n_q=(150, 1, 77), tails=(5, 0, 130), B=32),    # ragged batch, one empty view
    dict(ns=4, M=90, lens=(1, 40, 2, 0), n_q=(0, 90, 3, 0), tails=(3, 64, 0, 0), B=16),    # sessions without a token
    dict(ns=2, M=80, lens=(0, 0), n_q=(0, 0), tails=(0, 0)),                               # nobody has one
    dict(ns=2, M=300, lens=(20, 3), B=128, tails=(61, 127)),
    dict(M=200, B=256, lens=(2,), tails=(300,)),
    dict(M=130, lens=(30,), scale=0.02),
    dict(M=64, H=32, G=8, lens=(9,), tails=(11,)),
    # up to 64 tokens with many query rows, and one token fewer than that takes
    dict(M=64, H=64, G=8, lens=(9,), tails=(11,)),
    dict(M=56, H=64, G=8, lens=(0,), tails=(129,)),
    dict(M=55, H=64, G=8, lens=(5,), tails=(100,)),
    dict(ns=3, M=4, H=256, G=2, lens=(0, 3, 1), n_q=(4, 0, 3), tails=(3, 0, 200)),
]


@pytest.mark.parametrize("i", range(len(GEOMETRIES)))
def test_chunk_attention_matches_the_definition(i):
    c = Chunk(seed=10 * i, **GEOMETRIES[i])
    c.call()
    c.check()


# Items of several shares, CTAs with several items, the ring of tiles wrapped around many times when a masked tile comes up
LONG = [
    dict(M=700, H=16, G=4, lens=(300,), tails=(90,)),
    dict(ns=3, L=2, M=350, H=16, G=4, lens=(100, 33, 77), n_q=(350, 20, 111), tails=(50, 129, 0), B=32),
    dict(M=2500, H=8, G=2, lens=(0,), tails=(0,)),                     # causal part alone: items of 1 to 20 tiles
    dict(M=65, H=4, G=1, lens=(501,), tails=(10,)),                    # one KV head on all SMs
    dict(ns=9, M=129, H=8, G=8, lens=[5 * s for s in range(9)], n_q=[129 - 15 * s for s in range(9)], tails=(0, 200, 7)),
    dict(M=1111, H=6, G=2, lens=(17,), tails=(777,), B=80),
    # more keys and values than L2 holds: the line in two and in four parts a CTA
    dict(M=700, H=32, G=8, lens=(512,), tails=(40,)),
    dict(ns=2, M=450, H=32, G=8, lens=(1024, 500), n_q=(450, 449), tails=(3, 200)),
    dict(M=800, H=40, G=8, B=128, lens=(512,), tails=(127,)),
]


@pytest.mark.parametrize("i", range(len(LONG)))
def test_long_chunks(i):
    c = Chunk(seed=200 + i, **LONG[i])
    for _ in range(3):
        c.out.fill_(77.0); c.lse.fill_(55.0)
        c.call()
        c.check()


def test_many_sessions():
    ns = 101
    c = Chunk(ns=ns, H=8, G=2, B=16, lens=[(7 * s) % 23 if s % 5 else 0 for s in range(ns)], M=70, n_q=[(s * 13) % 71 for s in range(ns)],
              tails=[(11 * s) % 41 for s in range(ns)], seed=9)
    c.call()
    c.check()


def test_the_same_bits_from_run_to_run():
    c = Chunk(seed=3, **LONG[1])
    c.call()
    first = (c.out.clone(), c.lse.clone())
    for _ in range(10):
        c.call()
    assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


def test_a_chunk_in_parts_is_the_chunk():
    """The chunk's first tokens committed and the rest attended over them: the same definition, other tiles."""
    whole = Chunk(M=300, lens=(5,), tails=(20,), seed=5)
    whole.call()
    for lo, n in ((0, 100), (100, 1), (101, 199)):
        part = Chunk(M=n, lens=(5,), tails=(20 + lo,), seed=6)
        part.q, part.k, part.v = whole.q[:, lo:lo + n].contiguous(), whole.k, whole.v
        part.tk, part.tv = whole.tk.clone(), whole.tv.clone()
        part.call()
        part.check()
        a, b = part.lse, whole.lse[:, lo:lo + n]
        assert float((a - b).abs().max()) <= 2.0 ** -12
    whole.check()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_nothing_reaches_a_result_that_it_does_not_see(value):
    """Whatever the memory behind the view's end, behind the tail and in later tokens of the chunk holds."""
    kw = dict(ns=2, lens=(3, 5), B=32, M=150, n_q=(150, 77), tails=(9, 130), seed=3)
    c, clean = Chunk(**kw), Chunk(**kw)
    for s in range(2):
        c.k[s, :, :, c.lens[s] * c.B:] = value
        c.v[s, :, :, c.lens[s] * c.B:] = value
        end = c.tails[s] + c.n_q[s]
        c.tk[s, end:] = value
        c.tv[s, end:] = value
    at = 60                                                            # a token of the chunk: the ones before it stay clean
    for s in range(2):
        c.tk[s, c.tails[s] + at, :, 0, 5] = value
        c.tv[s, c.tails[s] + at, :, 1, 7] = value
    c.call()
    clean.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:, :at], clean.out[:, :at]) and torch.equal(c.lse[:, :at], clean.lse[:, :at])
    r = c.H // c.G
    # the value itself reaches exactly its own dim of the tokens from `at` on, in the heads that read it
    for s in range(2):
        for i in range(at, c.n_q[s]):
            got, want = c.out[s, i, 0, r:].float(), clean.out[s, i, 0, r:].float()
            same = torch.ones(D, dtype=torch.bool, device="cuda")
            same[7] = False
            assert torch.equal(got[:, same], want[:, same])
            assert bool(got[:, 7].isnan().all() if math.isnan(value) else (got[:, 7] == value).all())
    assert torch.equal(c.lse[:, :, :, r:], clean.lse[:, :, :, r:])
    c.guards.check()


def test_the_largest_values_do_not_overflow():
    """Values of 2^110 behind logits that grow from tile to tile: the weights before a reference moves are below 2^12, a product's sums
    below 2^122 times a few."""
    c, big = Chunk(lens=(24,), M=130, seed=8), Chunk(lens=(24,), M=130, seed=8)
    ramp = torch.linspace(0.1, 2.0, c.k.shape[3], device="cuda").view(1, 1, 1, -1, 1)
    for x in (c, big):
        x.k = (x.k.float() * ramp).to(torch.bfloat16)
    big.v, big.tv = big.v * 2.0 ** 110, big.tv * 2.0 ** 110
    c.call()
    big.call()
    torch.cuda.synchronize()
    assert torch.equal(big.out.float(), c.out.float() * 2.0 ** 110) and torch.equal(big.lse, c.lse)


@pytest.mark.parametrize("M,H,lens", [(140, 8, (3,)), (700, 16, (300,))])
def test_values_that_are_not_finite_in_the_last_tokens(M, H, lens):
    """In a share of an item that is joined later too: the last token's value is infinite in one dim."""
    kw = dict(M=M, H=H, G=2, lens=lens, seed=4)
    c, clean = Chunk(**kw), Chunk(**kw)
    c.tv[0, c.tails[0] + M - 1, :, :, 9] = math.inf
    c.call()
    clean.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out[0, :M - 1], clean.out[0, :M - 1])
    assert bool((c.out[0, M - 1, :, :, 9] == math.inf).all())
    same = torch.ones(D, dtype=torch.bool, device="cuda")
    same[9] = False
    assert torch.equal(c.out[0, M - 1][..., same], clean.out[0, M - 1][..., same])


def test_values_that_are_not_finite_in_many_short_items():
    """Every CTA with several items in turn, of one and of two row tiles, each with an infinite value at another token: it reaches the
    tokens from its own on and nothing else."""
    ns = 60
    kw = dict(ns=ns, H=16, G=8, B=16, M=150, lens=[(5 * s) % 19 for s in range(ns)], n_q=[150 - (17 * s) % 90 for s in range(ns)],
              tails=[(29 * s) % 150 for s in range(ns)], seed=13)
    c, clean = Chunk(**kw), Chunk(**kw)
    at = [(31 * s) % c.n_q[s] for s in range(ns)]
    for s in range(ns):
        c.tv[s, c.tails[s] + at[s], :, :, s] = math.inf
    clean.call()
    for _ in range(3):
        c.call()
        torch.cuda.synchronize()
        for s in range(ns):
            i, n = at[s], c.n_q[s]
            assert torch.equal(c.out[s, :i], clean.out[s, :i]), s
            assert bool((c.out[s, i:n, :, :, s] == math.inf).all()), s
            same = torch.ones(D, dtype=torch.bool, device="cuda")
            same[s] = False
            assert torch.equal(c.out[s, i:n][..., same], clean.out[s, i:n][..., same]), s
        assert torch.equal(c.lse, clean.lse)
    c.guards.check()


def test_large_logits_and_growing_maxima():
    """Keys that grow along the view, so that the running maximum moves in every tile; logits up to about 200."""
    c = Chunk(lens=(24,), M=130, seed=8, scale=0.5)
    ramp = torch.linspace(0.1, 4.0, c.k.shape[3], device="cuda").view(1, 1, 1, -1, 1)
    c.k = (c.k.float() * ramp).to(torch.bfloat16)
    c.call()
    c.check()


def test_rows_whose_logits_are_all_minus_infinity():
    c = Chunk(M=70, lens=(2,), seed=11)
    c.q[:, :, :, :4, 5] = 1.5
    c.k[:, :, 0, :, 5] = -math.inf
    c.tk[:, :, :, 0, 5] = -math.inf
    c.tv[:, c.tails[0] + 3, :, 0, 9] = math.inf
    c.call()
    torch.cuda.synchronize()
    assert bool((c.out[:, :, :, :4] == 0).all()) and bool((c.lse[:, :, :, :4] == -math.inf).all())
    assert bool(c.lse[:, :, :, 4:].isfinite().all())


def test_lengths_outside_the_tail_are_clamped_and_reported():
    c = Chunk(M=70, lens=(2,), tails=(5,), seed=12, tail_extra=0)
    c.nt_dev.fill_(5 + 40)
    c.call()
    c.check(status=kvmem.E_DEVICE_RANGE)
    c.nt_dev.fill_(-3)
    c.tails = [0]
    c.call()
    c.check(status=kvmem.E_DEVICE_RANGE)


def test_captured_and_replayed_with_other_lengths():
    """Lengths are the device's: a captured call follows them.  Two graphs with a workspace each run side by side."""
    kw = dict(ns=2, M=200, H=16, G=4, lens=(40, 13), n_q=(200, 90), tails=(9, 30), B=32)
    cs = [Chunk(seed=21 + i, **kw) for i in range(2)]
    graphs = []
    for c in cs:
        need = c.pool.lib.kvmem_prefill_workspace_bytes(c.pool.cfg, c.ns, c.M)
        c.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        c.call(workspace=c.ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(workspace=c.ws)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in cs]
    for n_q, lens in (((200, 90), (40, 13)), ((1, 200), (0, 40)), ((77, 0), (5, 1))):
        for c in cs:
            c.n_q, c.lens = list(n_q), list(lens)
            c.nq_dev.copy_(torch.tensor(n_q, dtype=torch.int32))
            c.n_sel.copy_(torch.tensor(lens, dtype=torch.int32))
            c.out.fill_(77.0); c.lse.fill_(55.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for c in cs:
            c.check()


def test_plain_launches():
    kvmem.set_option("pdl", 0)
    try:
        c = Chunk(seed=31, **LONG[0])
        c.call()
        c.check()
    finally:
        kvmem.set_option("pdl", 1)


def test_what_the_call_refuses():
    c = Chunk(M=70, lens=(2,), seed=1)
    view = View(c.k, c.v, c.capb * c.B)

    def refused(status, **kw):
        a = dict(q=c.q, view=view, n_sel=c.n_sel, tail=Tail(c.tk, c.tv, c.nt_dev), out=c.out, lse=c.lse)
        with pytest.raises(KvmemError) as e:
            c.pool.view_prefill_attend(**{**a, **kw})
        assert e.value.status == status, e.value

    refused(kvmem.E_INVALID, scale=-1.0)
    refused(kvmem.E_INVALID, scale=math.inf)
    refused(kvmem.E_CAPACITY, workspace=torch.empty(4096, dtype=torch.uint8, device="cuda"))
    short = Tail(c.tk[:, :69].contiguous(), c.tv[:, :69].contiguous(), c.nt_dev)
    refused(kvmem.E_INVALID, tail=short)
    for bad in (dict(q=c.q.float()), dict(out=c.out.float()), dict(n_q=c.nq_dev.long()), dict(lse=c.lse[:, :3]),
                dict(tail=Tail(c.tk, c.tv.float(), c.nt_dev)), dict(q=c.q.transpose(1, 3))):
        with pytest.raises(ValueError):
            c.pool.view_prefill_attend(**{**dict(q=c.q, view=view, n_sel=c.n_sel, tail=Tail(c.tk, c.tv, c.nt_dev), out=c.out, lse=c.lse), **bad})
    other = Pool(1, 8, 2, 64, 64, 1, 1, 1, torch.cuda.current_device())            # head_dim 64
    t = torch.zeros(1, 70, 1, 8, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(1, 1, 2, 128, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(KvmemError) as e:
        other.view_prefill_attend(t, View(kv, kv, 128), c.n_sel, None, t.clone(), torch.zeros(1, 70, 1, 8, device="cuda"))
    assert e.value.status == kvmem.E_UNSUPPORTED
    c.guards.check()
    assert bool((c.out == 77.0).all())
