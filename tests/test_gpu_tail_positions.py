"""Where the keys of a tail stand after commits and recalls, and what brings them to where the next tokens expect them.

A key in the tail keeps the position that it was turned to; a commit moves rows and no bits; positions of new tokens are counted from
rows.  Each way that kvmem_commit_blocks names is run over several rounds, and every key in the tail is compared with the definition: its
raw key turned, in 64 bits, to first_position + n_sel * block_tokens + its row.

Bounds.  A key turned once: `close` of the rotation's tests.  Turned again in place: the first rounding, at most 2^-8 of either element of
a pair, is turned with the pair, so it moves an element by at most 2^-8 of the pair's length (Cauchy-Schwarz), then the second
rounding, 2^-8 of the element; fp32 as in the first turn, 5 * 2^-24 of |a| + |b| <= sqrt(2) of the length, twice."""
import math

import pytest
import torch

from kvmem_harness import Guards
from paper_2609_04852_b200 import Rope, Tail
from test_gpu_tokens import close, dev, ints, make_pool, randn, to_pool_order, turned

pytestmark = pytest.mark.gpu
L, H, G, B, D, NS = 2, 8, 2, 32, 128, 2
ROPES = [Rope(), Rope("interleaved", 96, "ramp", 4.0, 512.0)]


class Loop:
    """Two sessions that have 5 committed blocks, a view of three of them at `first`, and 70 tokens in the tail behind it."""

    def __init__(self, rope, first=17, seed=0):
        self.rope, self.first = rope, first
        self.pool = make_pool(L, H, G, D, B, NS, 12, 2048, rope)
        self.k, self.v = randn(seed, NS, 400, L, G, D), randn(seed + 1, NS, 400, L, G, D)
        self.q = randn(seed + 2, NS, 400, L, H, D)
        self.raw = self.k[..., to_pool_order(rope, D)]
        self.guards = Guards(dev())
        self.cap = 200
        self.tail = Tail(*(self.guards.empty((NS, self.cap, L, G, D), torch.bfloat16, fill=3.0) for _ in range(2)), ints([0] * NS))
        self.at, self.front = 0, 0                          # tokens so far; the token in row 0
        self.sel, self.n_sel = torch.zeros(NS, 12, dtype=torch.int32, device="cuda"), ints([0] * NS)
        self.view = self.pool.new_view(NS, 12 * B)
        for s in range(NS):
            self.pool.reserve_blocks(s, 12)
        self.append(5 * B)
        self.commit(5)
        assert self.tail.n_tokens.tolist() == [0] * NS
        self.recall([[0, 2, 4]] * NS)
        self.append(70)

    def append(self, m, pages=True, **kw):
        rows = slice(self.at, self.at + m)
        self.q_out = torch.zeros(NS, m, L, H, D, dtype=torch.bfloat16, device="cuda")
        self.pool.append_tokens(self.k[:, rows], self.v[:, rows], self.tail, q=self.q[:, rows], q_out=self.q_out, n_sel=self.n_sel,
                                pages=pages, **{**dict(first_position=self.first), **kw})
        self.tail.n_tokens += m
        self.at += m

    def commit(self, n):
        self.pool.commit_blocks([n] * NS, self.tail)
        self.front += n * B

    def recall(self, ids):
        for s, x in enumerate(ids):
            self.sel[s, :len(x)] = ints(x)
        self.n_sel.copy_(ints([len(x) for x in ids]))
        self.pool.materialize_rope(self.sel, self.n_sel, self.view, self.first)

    def check(self, turns=1, offset=0):
        """Every token of the tail stands at first_position + n_sel * block_tokens + offset + its row."""
        torch.cuda.synchronize()
        n = self.at - self.front
        assert self.pool.device_status() == 0 and self.tail.n_tokens.tolist() == [n] * NS
        for s in range(NS):
            pos = self.first + int(self.n_sel[s]) * B + offset + torch.arange(n, device="cuda").view(n, 1, 1)
            ref, mag = turned(self.raw[s, self.front:self.at].double(), pos, self.rope)
            got = self.tail.k[s, :n]
            if turns == 1:
                close(got, ref, mag)
            else:
                m = (self.rope.rotary_dim or D) // 2
                length = torch.zeros_like(ref)
                length[..., :m] = length[..., D // 2:D // 2 + m] = (ref[..., :m] ** 2 + ref[..., D // 2:D // 2 + m] ** 2).sqrt()
                tol = (2.0 ** -8 * length + 2.0 ** -8 * ref.abs() + 2 * 5 * 2.0 ** -24 * math.sqrt(2.0) * length) * (1 + 2.0 ** -7)
                assert bool(((got.double() - ref).abs() <= tol).all())
            assert torch.equal(self.tail.v[s, :n], self.v[s, self.front:self.at])
        self.guards.check()

    def turn(self, difference):
        """The tail's keys of each session, turned in place by its difference."""
        for back in (False, True):
            by = [max(-x if back else x, 0) for x in difference]
            if any(by):
                x = self.tail.k.view(NS * self.cap, L * G, D)
                self.pool.rope_apply(x, ints(by).repeat_interleave(self.cap), out=x, inverse=back, x_order="pool", out_order="pool")

    def attends(self):
        """The last appended tokens over view and tail, as the model would: relative to positions in 64 bits, mean error against mean size."""
        m = self.q_out.shape[1]
        out, lse = torch.zeros_like(self.q_out), torch.zeros(NS, m, L, H, device="cuda")
        self.tail.n_tokens -= m
        self.pool.view_prefill_attend(self.q_out, self.view, self.n_sel, self.tail, out, lse)
        self.tail.n_tokens += m
        order = to_pool_order(self.rope, D)
        for s in range(NS):
            ids = self.sel[s, :int(self.n_sel[s])].tolist()
            tok = torch.cat([torch.arange(b * B, (b + 1) * B) for b in ids] + [torch.arange(self.front, self.at)]).cuda()
            pos = self.first + torch.arange(tok.numel(), device="cuda")
            K, V = turned(self.raw[s, tok].double(), pos.view(-1, 1, 1), self.rope)[0], self.v[s, tok].double()
            Q = turned(self.q[s, self.at - m:self.at][..., order].double(), pos[-m:].view(-1, 1, 1), self.rope)[0]
            x = torch.einsum("ilgrd,jlgd->lgrij", Q.view(m, L, G, H // G, D), K) / math.sqrt(D)
            x = torch.where(torch.arange(tok.numel(), device="cuda") <= (tok.numel() - m + torch.arange(m, device="cuda")).view(-1, 1), x, -math.inf)
            ref = torch.einsum("lgrij,jlgd->ilgrd", torch.softmax(x, -1), V).reshape(m, L, H, D)
            err = (out[s].double() - ref).abs()
            assert err.mean().item() < 0.02 * ref.abs().mean().item()


@pytest.mark.parametrize("rope", ROPES)
def test_a_commit_keeps_the_keys_where_they_were(rope):
    """What the header says of the bits, and what it warns of: counted from rows, new tokens come in front of older ones."""
    c = Loop(rope)
    c.check()
    before = c.tail.k.clone()
    c.commit(2)
    assert torch.equal(c.tail.k[:, :6], before[:, 64:70])
    c.check(offset=2 * B)                                   # row r: where row r + 64 was
    c.append(5)
    ref, mag = turned(c.raw[0, c.at - 5:c.at].double(), (c.first + 3 * B + 6 + torch.arange(5, device="cuda")).view(-1, 1, 1), rope)
    close(c.tail.k[0, 6:11], ref, mag)                      # 58 positions in front of the token before them


@pytest.mark.parametrize("rope", ROPES)
def test_a_view_that_grows_by_the_committed_blocks(rope):
    c = Loop(rope)
    for ids in ([0, 2, 4, 5, 6], [0, 2, 4, 5, 6, 7]):
        c.commit(len(ids) - int(c.n_sel[0]))
        c.recall([ids] * NS)
        c.check()
        c.append(40)
        c.check()
        c.attends()


@pytest.mark.parametrize("rope", ROPES)
def test_a_view_that_stays(rope):
    """New tokens go on behind the tail's, over the gap that the committed ones leave."""
    c = Loop(rope)
    gone = 0
    for n in (2, 1):
        c.commit(n)
        gone += n * B
        c.append(40, first_position=c.first + gone)
        c.check(offset=gone)
    # the same by positions
    c.append(3, positions=ints([[c.first + 3 * B + gone + c.at - c.front + i for i in range(3)]] * NS))
    c.check(offset=gone)


@pytest.mark.parametrize("rope", ROPES)
def test_keys_turned_by_the_difference(rope):
    """Other views, shorter and longer, other ones for each session; one more rounding."""
    c = Loop(rope)
    was = [c.first + 3 * B + 2 * B] * NS
    c.commit(2)
    c.recall([[1], [0, 3, 5, 6]])
    c.turn([c.first + int(n) * B - w for n, w in zip(c.n_sel, was)])
    c.check(turns=2)
    c.append(9)
    c.check(turns=2)
    c.attends()
    d = Loop(rope)
    d.commit(1)
    d.recall([[0, 1, 2, 3, 4, 5], [5]])
    d.turn([(6 - 3 - 1) * B, (1 - 3 - 1) * B])
    d.check(turns=2)
    d.append(9)
    d.check(turns=2)


@pytest.mark.parametrize("rope", ROPES)
def test_raw_keys_appended_again(rope):
    """No second rounding, whatever the views were."""
    c = Loop(rope)
    for n, ids in ((2, [[1], [0, 3, 5, 6]]), (1, [[0, 1, 2, 3, 4, 5, 6], [7]])):
        c.commit(n)
        c.recall(ids)
        held = c.at - c.front
        c.at = c.front
        c.tail.n_tokens.zero_()
        c.append(held, pages=False)
        c.check()
        c.append(40)
        c.check()
        c.attends()
