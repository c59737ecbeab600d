"""New tokens on their way into the cache: rotary forms, rows of the tail and of reserved pages, commits; and the whole loop with a
model whose rotary form is not the pool's.

Bounds.  A rotated element is amplitude (a cos - b sin): cos and sin are off by at most 2^-24 (one rounding of the 64-bit value),
two products, a sum and the amplitude's product are rounded to fp32, 2^-24 each of at most |a| + |b|: 5 * 2^-24 amplitude (|a| + |b|); then
one rounding to bf16, 2^-8 of the result.  Dims that pass, values and raw keys are copies: equal bits."""
import ctypes as C
import math

import pytest
import torch

from kvmem_harness import Guards
from paper_2609_04852_b200 import KvmemError, Pool, Rope, SelectParams, Tail
from paper_2609_04852_b200 import kvmem

pytestmark = pytest.mark.gpu
THETA = 1.0e4


def dev():
    return torch.device("cuda", torch.cuda.current_device())


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------------------

def frequencies(rope, d, theta=THETA):
    n = rope.rotary_dim or d
    out = []
    fast = rope.turns_fast or (32.0 if rope.scaling == "ramp" else 4.0)
    slow = rope.turns_slow or 1.0
    for i in range(n // 2):
        f = theta ** (-2.0 * i / n)
        if rope.scaling == "linear":
            f /= rope.factor
        elif rope.scaling == "base":
            f = (theta * rope.factor ** (n / (n - 2))) ** (-2.0 * i / n)
        elif rope.scaling == "ramp":
            p = lambda t: n * math.log(rope.original_positions / (2 * math.pi * t)) / (2 * math.log(theta))
            lo, hi = max(math.floor(p(fast)), 0), min(math.ceil(p(slow)), n - 1)
            x = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = f / rope.factor * x + f * (1 - x)
        elif rope.scaling == "bands":
            x = min(max((fast - rope.original_positions * f / (2 * math.pi)) / (fast - slow), 0.0), 1.0)
            f = f / rope.factor * x + f * (1 - x)
        out.append(f)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def to_pool_order(rope, d):
    """index: the model's dim that stands at each of the pool's."""
    n = rope.rotary_dim or d
    a, b = (range(0, n // 2), range(n // 2, n)) if rope.layout == "half" else (range(0, n, 2), range(1, n, 2))
    rest = list(range(n, d))
    h = (d - n) // 2
    return torch.tensor(list(a) + rest[:h] + list(b) + rest[h:], device="cuda")


def turned(x, positions, rope, theta=THETA, sign=1.0, amplitude=1.0):
    """x fp64 [..., d] in the pool's order, positions broadcastable to its leading dims: (result, |a| + |b| of every element)."""
    d = x.shape[-1]
    n = (rope.rotary_dim or d) // 2
    ang = positions.double().unsqueeze(-1) * frequencies(rope, d, theta)
    c, s = ang.cos(), sign * ang.sin()
    a, b = x[..., :n], x[..., d // 2:d // 2 + n]
    y, mag = x.clone(), torch.zeros_like(x)
    y[..., :n] = amplitude * (a * c - b * s)
    y[..., d // 2:d // 2 + n] = amplitude * (b * c + a * s)
    mag[..., :n] = mag[..., d // 2:d // 2 + n] = amplitude * (a.abs() + b.abs())
    return y, mag


def close(got, ref, mag):
    tol = 2.0 ** -8 * ref.abs() + (1 + 2.0 ** -8) * 5 * 2.0 ** -24 * mag
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), (err - tol).max().item()


FORMS = [
    Rope(),
    Rope("interleaved"),
    Rope("half", 64),
    Rope("interleaved", 32, "linear", 3.0),
    Rope("half", 112, "base", 4.0),
    Rope("interleaved", 96, "ramp", 8.0, 512.0),
    Rope("half", 0, "bands", 8.0, 300.0),
    Rope("half", 0, "ramp", 2.0, 1000.0, 16.0, 2.0),
    Rope("interleaved", 16, "bands", 2.0, 64.0, 3.0, 0.5),
]


def make_pool(L=1, H=8, G=2, d=128, B=64, ns=1, blocks=4, positions=4096, rope=None, **kw):
    pool = Pool(L, H, G, d, B, ns, max(1, ns * blocks), max(1, blocks), dev().index, rope_max_positions=positions,
                rope_theta=THETA if positions else 0.0, **kw)
    if rope is not None:
        pool.set_rope(rope)
    return pool


def test_frequencies_of_every_form():
    pool = make_pool()
    for rope in FORMS:
        f, n = pool.rope_frequencies(rope), (rope.rotary_dim or 128) // 2
        want = frequencies(rope, 128).tolist()
        assert all(abs(x - y) <= 1e-14 * y for x, y in zip(f[:n], want)) and f[n:] == [0.0] * (64 - n), rope
    assert pool.rope_frequencies() == pool.rope_frequencies(Rope())


# ---- rotation -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("i", range(len(FORMS)))
@pytest.mark.parametrize("orders", [("model", "pool"), ("model", "model"), ("pool", "pool"), ("pool", "model")])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_matches_the_definition(i, orders, inverse):
    rope = FORMS[i]
    pool = make_pool(rope=rope)
    rows, heads, amplitude = 37, 1 + i, 1.0 if i % 2 else 1.25
    x = randn(i, rows, heads, 128)
    pos = torch.randint(0, 4096, (rows,), generator=torch.Generator().manual_seed(i)).to(torch.int32).cuda()
    pos[0], pos[1] = 0, 4095
    guards = Guards(dev())
    out = guards.empty((rows, heads, 128), torch.bfloat16, fill=9.0)
    got = pool.rope_apply(x, pos, out=out, inverse=inverse, amplitude=amplitude, x_order=orders[0], out_order=orders[1])
    assert got is out and pool.device_status() == 0
    order = to_pool_order(rope, 128)
    xp = x.double() if orders[0] == "pool" else x.double()[..., order]
    ref, mag = turned(xp, pos.view(-1, 1), rope, sign=-1.0 if inverse else 1.0, amplitude=amplitude)
    gp = out if orders[1] == "pool" else out[..., order]
    close(gp, ref, mag)
    n = (rope.rotary_dim or 128) // 2
    rest = torch.ones(128, dtype=torch.bool, device="cuda")
    rest[:n] = False
    rest[64:64 + n] = False
    assert torch.equal(gp[..., rest].double(), xp[..., rest])
    guards.check()


@pytest.mark.parametrize("d,rotary", [(16, 0), (16, 16), (32, 16), (64, 48), (80, 32), (96, 96), (256, 64), (256, 0), (512, 240)])
def test_rotation_of_other_head_dims(d, rotary):
    rope = Rope("interleaved", rotary)
    pool = make_pool(H=1, G=1, d=d, rope=rope)
    x = randn(d, 129, 3, d)
    pos = (torch.arange(129) * 31 % 4096).to(torch.int32).cuda()
    out = pool.rope_apply(x, pos)
    assert pool.device_status() == 0
    ref, mag = turned(x.double()[..., to_pool_order(rope, d)], pos.view(-1, 1), rope)
    close(out, ref, mag)


def test_rotation_of_strided_vectors():
    rope = Rope("interleaved", 64)
    pool = make_pool(rope=rope)
    pos = (torch.arange(300) * 13).to(torch.int32).cuda()
    wide = randn(1, 300, 50 * 128)
    x = wide[:, 5 * 128:45 * 128].unflatten(1, (40, 128))                      # a slice of a packed projection
    plain = pool.rope_apply(x.contiguous(), pos)
    assert torch.equal(pool.rope_apply(x, pos), plain)
    heads_first = torch.zeros(40, 300, 128, dtype=torch.bfloat16, device="cuda")
    pool.rope_apply(x, pos, out=heads_first.transpose(0, 1))                   # vectors outside, rows inside
    assert torch.equal(heads_first.transpose(0, 1), plain)
    one = x[:, :1].expand(300, 6, 128)                                         # one head for many: stride 0
    assert torch.equal(pool.rope_apply(one, pos), plain[:, :1].expand(300, 6, 128))
    before = wide.clone()
    same = pool.rope_apply(x, pos, out_order="model")
    pool.rope_apply(x, pos, out=x, out_order="model")                          # in place
    assert torch.equal(x, same)
    before[:, 5 * 128:45 * 128] = same.flatten(1)
    assert torch.equal(wide, before), "elements beside the slice were written"
    assert pool.device_status() == 0


def test_there_and_back_and_the_gradient():
    """Back is the transpose of there (the gradient of a scalar product), and undoes it to two roundings."""
    rope = Rope("half", 96, "ramp", 4.0, 512.0)
    pool = make_pool(rope=rope)
    pos = (torch.arange(64) * 61).to(torch.int32).cuda()
    x, g = randn(1, 64, 4, 128), randn(2, 64, 4, 128)
    y = pool.rope_apply(x, pos)
    back = pool.rope_apply(y, pos, inverse=True, x_order="pool", out_order="model")
    err = (back.double() - x.double()).abs()
    pair = x.double()[..., to_pool_order(rope, 128)]
    size = (pair[..., :64] ** 2 + pair[..., 64:] ** 2).sqrt().max().item()
    assert err.max().item() <= 2 * 2.0 ** -8 * size * math.sqrt(2.0) * 1.01        # each rounding moves either element of a pair
    dx = pool.rope_apply(g, pos, inverse=True, x_order="pool", out_order="model")
    lhs, rhs = (g.double() * y.double()).sum(-1), (dx.double() * x.double()).sum(-1)
    tol = 2.0 ** -8 * ((g.double() * y.double()).abs().sum(-1) + (dx.double() * x.double()).abs().sum(-1)) * 1.01
    assert bool(((lhs - rhs).abs() <= tol).all())


def test_the_pools_own_form_is_rope_rotate():
    """The same arithmetic; the table that set_rope builds differs from the one a pool is created with by the last bit of a 64-bit
    cosine at most, which one entry in 2^28 or so would round to another fp32."""
    pool = make_pool()
    x, pos = randn(3, 500, 8, 128), torch.arange(0, 4000, 8).to(torch.int32).cuda()
    a = pool.rope_rotate(x, pos)
    assert torch.equal(pool.rope_apply(x, pos), a)
    assert torch.equal(pool.rope_apply(x, pos, inverse=True), pool.rope_rotate(x, pos, inverse=True))
    pool.set_rope(Rope("interleaved", 64, "linear", 2.0))
    assert not torch.equal(pool.rope_rotate(x, pos), a)
    pool.set_rope()
    b = pool.rope_rotate(x, pos)
    assert int((a != b).sum()) <= 8


def test_positions_outside_the_table_are_left_out():
    pool = make_pool(positions=100, rope=Rope("interleaved"))
    pos = ints([5, -1, 99, 100, 2 ** 31 - 1, -2 ** 31, 0])
    out = torch.full((7, 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    pool.rope_apply(randn(1, 7, 3, 128), pos, out=out)
    assert pool.device_status() == kvmem.E_DEVICE_RANGE and pool.device_status() == 0
    left = (out == 7.0).all(2).all(1).tolist()
    assert left == [False, True, False, True, True, True, False]


def test_far_positions():
    """Angles of up to 10^6 radians: exact to fp32 in the table."""
    rope = Rope("half", 0, "linear", 1.0)
    pool = make_pool(H=1, G=1, d=64, positions=1000003, rope=rope)
    pos = ints([1000002, 999999, 524288, 777777])
    x = randn(5, 4, 2, 64)
    ref, mag = turned(x.double(), pos.view(-1, 1), rope)
    # (a 64-bit angle of 10^6 is good to 10^-10)
    close(pool.rope_apply(x, pos), ref, mag * (1 + 1e-3))


def test_what_rotation_refuses():
    pool = make_pool(rope=Rope("interleaved", 64))
    x, pos = randn(1, 10, 4, 128), torch.arange(10, dtype=torch.int32, device="cuda")
    lib, st = pool.lib, torch.cuda.current_stream().cuda_stream

    def call(**kw):
        a = dict(x=x.data_ptr(), xr=512, xv=128, xo=0, y=x.data_ptr() + (1 << 40), yr=512, yv=128, yo=1, n=10, v=4, p=pos.data_ptr(), inv=0, amp=1.0)
        a["y"] = out.data_ptr()
        a.update(kw)
        return lib.kvmem_rope_apply(pool.handle, a["x"], a["xr"], a["xv"], a["xo"], a["y"], a["yr"], a["yv"], a["yo"], a["n"], a["v"], a["p"], a["inv"], a["amp"], st)

    out = torch.full((10, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(x=None), dict(p=None), dict(x=x.data_ptr() + 2), dict(xr=511), dict(yv=-128), dict(v=0), dict(n=-1), dict(xo=2), dict(yo=-1),
               dict(amp=math.nan), dict(amp=-1.0), dict(yr=128), dict(yv=64), dict(yv=0), dict(y=x.data_ptr()), dict(y=x.data_ptr() + 64, yo=0),
               dict(y=x.data_ptr(), yo=0, yr=1024), dict(y=x.data_ptr() + 2 * 5 * 512, yo=0)):
        assert call(**kw) == kvmem.E_INVALID, kw
    assert call(n=0, x=None) == kvmem.OK
    for bad in (Rope("half", 8), Rope("half", 100)):
        with pytest.raises(KvmemError) as e:
            pool.set_rope(bad)
        assert e.value.status == kvmem.E_UNSUPPORTED
    for bad in (Rope("half", 144), Rope("half", -16), Rope("half", 0, "linear", 0.5), Rope("half", 0, "base", math.inf), Rope("half", 0, "ramp", 2.0),
                Rope("half", 0, "bands", 2.0, 100.0, 1.0, 2.0), Rope("half", 0, "bands", 2.0, math.nan), Rope("half", 0, "ramp", 2.0, 100.0, 4.0, -1.0)):
        with pytest.raises(KvmemError) as e:
            pool.set_rope(bad)
        assert e.value.status == kvmem.E_INVALID, bad
    for bad in (Rope("thirds"), Rope("half", 0, "magic")):
        with pytest.raises(ValueError):
            pool.set_rope(bad)
    for kw in (dict(x_order="mine"), dict(out=out[:, :2]), dict(out=out.float())):
        with pytest.raises(ValueError):
            pool.rope_apply(x, pos, **kw)
    with pytest.raises(ValueError):
        pool.rope_apply(x, pos.long())
    with pytest.raises(ValueError):
        pool.rope_apply(x[..., ::2], pos)
    plain = make_pool(positions=0)
    for f in (lambda: plain.set_rope(Rope()), lambda: plain.rope_apply(x, pos), lambda: plain.rope_frequencies()):
        with pytest.raises(KvmemError) as e:
            f()
        assert e.value.status == kvmem.E_STATE
    k = randn(2, 64, 1, 2, 128)
    pool.append_blocks(0, k, k)
    with pytest.raises(KvmemError) as e:
        pool.set_rope(Rope())
    assert e.value.status == kvmem.E_STATE
    pool.session_reset(0)
    pool.reserve_blocks(0, 1)
    with pytest.raises(KvmemError) as e:
        pool.set_rope(Rope())
    assert e.value.status == kvmem.E_STATE
    pool.session_reset(0)
    pool.set_rope(Rope())
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("in_block", [False, True])
@pytest.mark.parametrize("i", [1, 2, 5, 6])
def test_every_pass_rotates_by_the_pools_form(i, in_block):
    """Materialised, fused, copy-free and cached views of a pool with a model's form: keys as the definition has them from raw keys in
    the pool's order, and the attention of each pass is that over the keys it wrote or would write.

    Bounds: a key of the materialised view on raw pages is one rotation (`close`), with in-block keys two roundings more of at most
    2^-8 of the pair each.  Attention results are compared with one another at the 2e-3 of the other passes' tests (unit-scale values;
    one bf16 step of some keys apart)."""
    rope, B, NB, G, H = FORMS[i], 64, 12, 2, 8
    pool = make_pool(1, H, G, B=B, blocks=NB, positions=2048, rope=rope, rope_in_block_keys=in_block)
    raw = randn(i, NB * B, 1, G, 128)                                       # the pool's order
    v = randn(50 + i, NB * B, 1, G, 128)
    # as a prefill left them: rotated at positions of their own, block by block
    pos0 = [(37 * b) % 1900 for b in range(NB)]
    at = torch.cat([torch.arange(p, p + B) for p in pos0]).to(torch.int32).cuda()
    roped = pool.rope_apply(raw[:, 0], at, x_order="pool")
    pool.append_blocks_rope(0, roped.unsqueeze(1).contiguous(), v, pos0)
    back = pool.rope_apply(roped, at, inverse=True, x_order="pool", out_order="pool")        # what the pages hold or are made from
    kbar = torch.zeros(NB, G, 128, device="cuda")
    for t in range(B):
        kbar = kbar + back.view(NB, B, G, 128)[:, t].float()
    assert torch.equal(pool.index(0)[0].transpose(0, 1), (kbar * (1.0 / B)).to(torch.bfloat16))
    sel, n_sel = ints([[0, 3, 4, 9, 11]]), ints([5])
    first = 100
    view = pool.new_view(1, 5 * B)
    pool.materialize_rope(sel, n_sel, view, first)
    keys = torch.cat([back.view(NB, B, G, 128)[b] for b in sel[0].tolist()]).double()
    where = (first + torch.arange(5 * B, device="cuda")).view(-1, 1)
    ref, mag = turned(keys, where, rope)
    got = view.k[0, 0].transpose(0, 1).double()
    if in_block:
        # the stored key is a rounded rotation, and its rotation is rounded: 2^-8 of an element's pair each
        n = (rope.rotary_dim or 128) // 2
        size = mag.clone()
        size[..., n:64] = keys[..., n:64].abs()
        size[..., 64 + n:] = keys[..., 64 + n:].abs()
        assert bool(((got - ref).abs() <= 2 * 2.0 ** -8 * size * 1.02 + 1e-30).all())
    else:
        close(view.k[0, 0].transpose(0, 1), ref, mag)
    q = pool.rope_apply(randn(90 + i, 3, H, 128), ints([first + 5 * B] * 3)).view(1, 3, 1, H, 128)
    outs = [pool.new_outputs(1, 3) for _ in range(4)]
    pool.view_attend(q, view, n_sel, *outs[0])
    pool.paged_attend_rope(q, sel, n_sel, *outs[1], first_position=first)
    view2 = pool.new_view(1, 5 * B)
    pool.materialize_attend_rope(q, sel, n_sel, view2, *outs[2], first_position=first)
    n_out = 3
    if not in_block:
        cache = pool.new_view_cache(5, 2, first)
        cache.update(0, ints([0, 1, 2, 9, 11]), n_sel)
        cache.update(0, sel[0].contiguous(), n_sel)                         # two blocks keep their slots and turn on by a delta
        cache.attend(q[0], outs[3][0][0], outs[3][1][0])
        n_out = 4
    assert torch.equal(view2.v, view.v)
    for o, l in outs[1:n_out]:
        assert float((o - outs[0][0]).abs().max()) <= 2e-2 and float((l - outs[0][1]).abs().max()) <= 2e-2
    # and they follow the positions: the same keys a few positions on are others
    pool.materialize_rope(sel, n_sel, view2, first + 5)
    assert not torch.equal(view2.k, view.k)
    assert pool.device_status() == 0


# ---- append ---------------------------------------------------------------------------------------------------------------------

class Append:
    """One append's inputs, buffers between guard bytes, and the 64-bit result."""

    def __init__(self, ns=1, L=1, H=8, G=2, d=128, B=64, M=5, n_new=None, tails=(7,), sel=(3,), first=0, rope=Rope(), positions=4096, pages=True,
                 queries=True, explicit=False, amplitude=1.0, seed=0, extra=2, packed=True):
        self.__dict__.update(ns=ns, L=L, H=H, G=G, d=d, B=B, M=M, first=first, rope=rope, window=positions, pages=pages, amplitude=amplitude)
        self.n_new = [M] * ns if n_new is None else list(n_new)
        self.tails = [tails[s % len(tails)] for s in range(ns)]
        self.sel = [sel[s % len(sel)] for s in range(ns)] if sel is not None else None
        self.cap = max(self.tails) + M + extra
        self.per = (self.cap + B - 1) // B
        self.pool = make_pool(L, H, G, d, B, ns, self.per + 1, positions, rope if positions else None)
        x = randn(seed, ns, M, L, H + 2 * G, d)
        self.q, self.k, self.v = x[..., :H, :], x[..., H:H + G, :], x[..., H + G:, :]
        if not packed:
            self.q, self.k, self.v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (self.q, self.k, self.v))
        if not queries:
            self.q = None
        self.positions = None
        if explicit:
            self.positions = torch.randint(0, positions, (ns, M), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.guards = Guards(dev())
        fill = dict(fill=5.0)
        self.tail = Tail(self.guards.empty((ns, self.cap, L, G, d), torch.bfloat16, **fill), self.guards.empty((ns, self.cap, L, G, d), torch.bfloat16, **fill),
                         ints(self.tails))
        self.q_out = self.guards.empty((ns, M, L, H, d), torch.bfloat16, **fill) if queries else None
        self.pool.pages().fill_(4.0)
        self.table = torch.randperm(ns * (self.per + 1), generator=torch.Generator().manual_seed(seed))[:ns * self.per].view(ns, self.per)
        if pages:
            for s in range(ns):
                self.pool.reserve_blocks(s, self.per, self.table[s].tolist())

    def call(self, **kw):
        a = dict(q=self.q, q_out=self.q_out, n_new=ints(self.n_new), positions=self.positions, n_sel=None if self.sel is None else ints(self.sel),
                 first_position=self.first, q_amplitude=self.amplitude, pages=self.pages)
        self.pool.append_tokens(self.k, self.v, self.tail, **{**a, **kw})

    def check(self, status=0):
        torch.cuda.synchronize()
        assert self.pool.device_status() == status
        d, order = self.d, to_pool_order(self.rope, self.d) if self.window else torch.arange(self.d, device="cuda")
        want_pages = torch.full_like(self.pool.pages(), 4.0)
        for s in range(self.ns):
            n, t = self.n_new[s], self.tails[s]
            pos = (t + torch.arange(n, device="cuda") + self.first + (self.sel[s] * self.B if self.sel is not None else 0)) if self.positions is None else self.positions[s, :n]
            raw = self.k[s, :n][..., order]
            rows = [(self.tail.k[s, t:t + n], raw, 1.0)]
            if self.q is not None:
                rows.append((self.q_out[s, :n], self.q[s, :n][..., order], self.amplitude))
                assert bool((self.q_out[s, n:] == 5.0).all())
            for got, x, amp in rows:
                if not self.window:
                    assert torch.equal(got, x)
                    continue
                close(got, *turned(x.double(), pos.view(-1, 1, 1), self.rope, amplitude=amp))
            assert torch.equal(self.tail.v[s, t:t + n], self.v[s, :n])
            for x in (self.tail.k, self.tail.v):
                assert bool((x[s, :t] == 5.0).all()) and bool((x[s, t + n:] == 5.0).all()), "rows that are not new were written"
            if self.pages:
                for i in range(n):
                    b, o = divmod(t + i, self.B)
                    want_pages[self.table[s, b], 0, :, :, o], want_pages[self.table[s, b], 1, :, :, o] = raw[i], self.v[s, i]
        assert torch.equal(self.pool.pages(), want_pages)
        assert self.tail.n_tokens.tolist() == self.tails
        self.guards.check()


APPENDS = [
    dict(),
    dict(M=1, tails=(0,)),                                             # a single token, an empty tail
    dict(M=1, H=1, G=1, tails=(63,), rope=Rope("interleaved")),        # the block's last token
    dict(M=70, tails=(60,), rope=Rope("half", 64)),                    # over a block's end
    dict(M=200, B=16, tails=(3,), rope=Rope("interleaved", 96, "ramp", 8.0, 512.0)),
    dict(ns=3, L=2, M=9, n_new=(9, 0, 4), tails=(5, 0, 130), B=32, sel=(1, 0, 9), first=100, rope=Rope("interleaved", 32)),
    dict(ns=40, M=1, tails=(0, 17, 63, 64, 128), sel=(0, 7, 20)),      # a decode step of many sessions
    dict(M=6, queries=False, rope=Rope("interleaved")),                # keys and values alone
    dict(M=33, pages=False, tails=(900,), amplitude=1.75, rope=Rope("half", 16, "linear", 4.0)),
    dict(ns=2, M=12, explicit=True, tails=(1, 40), rope=Rope("interleaved", 0, "bands", 8.0, 300.0)),
    dict(M=21, positions=0, sel=None),                                 # no rotary support: copies
    dict(M=10, d=64, H=5, G=5, B=48, rope=Rope("interleaved", 48), sel=None),
    dict(M=10, d=256, H=6, G=2, rope=Rope("half", 64, "base", 2.0)),
    dict(ns=4, M=30, packed=False, tails=(2, 9), rope=Rope("interleaved")),
    dict(M=1500, L=3, H=12, G=4, tails=(100,), rope=Rope("interleaved", 128), sel=None),
]


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append_matches_the_definition(i):
    c = Append(seed=i, **APPENDS[i])
    c.call()
    c.check()
    c.call()                                                           # again: the same tokens in the same rows
    c.check()


def test_append_all_rows_without_counts():
    c = Append(ns=2, M=6, tails=(1, 2))
    c.call(n_new=None)
    c.check()


def test_tail_lengths_outside_the_tail_are_clamped_and_reported():
    c = Append(M=6, tails=(5,), extra=0, pages=False)
    c.tail.n_tokens.fill_(100)
    c.call()
    c.tail.n_tokens.fill_(5)
    c.check(status=kvmem.E_DEVICE_RANGE)
    c = Append(M=6, tails=(0,), pages=False)
    c.tail.n_tokens.fill_(-9)
    c.call()
    c.tail.n_tokens.fill_(0)
    c.check(status=kvmem.E_DEVICE_RANGE)


def test_tokens_at_positions_outside_the_table_are_left_out():
    c = Append(ns=2, M=6, tails=(3,), positions=200, sel=(2,), first=60)         # 60 + 128 + 3 + i
    c.call(first_position=66)                                                   # 197 .. 202
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE
    for x in (c.tail.k[:, 3:], c.tail.v[:, 3:], c.q_out):
        assert bool((x[:, 3:6] == 5.0).all()) and not bool((x[:, :3] == 5.0).all(-1).any())
    c.guards.check()


def test_rows_without_a_reserved_page():
    """Nothing is written to pages that the session has not got, whatever earlier sessions left in the table."""
    c = Append(ns=2, M=100, tails=(0,), pages=False)
    k = randn(9, 128, 1, 2, 128)
    c.pool.append_blocks(0, k, k)
    c.pool.session_reset(0)
    c.pool.append_blocks(1, k, k)                                       # the pages that session 0 had
    c.pool.reserve_blocks(0, 1)
    table = c.pool.block_table(1).tolist()
    before = c.pool.pages().clone()
    c.call(pages=True, first_position=0)
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE
    assert torch.equal(c.tail.v[:, :100], c.v)                          # the tail is complete
    after = c.pool.pages()
    changed = [p for p in range(after.shape[0]) if not torch.equal(after[p], before[p])]
    assert len(changed) == 1 and changed[0] not in table                # session 0's reserved page; session 1 reserved none
    assert torch.equal(after[changed[0], 1, 0], c.v[0, :64, 0].transpose(0, 1))


@pytest.mark.parametrize("B,rope", [(16, None), (64, Rope("interleaved", 64)), (48, Rope("half"))])
def test_token_by_token_is_block_by_block(B, rope):
    """Appending in any steps and committing gives the pages, the index and the table that appending whole blocks gives."""
    L, G, n = 2, 2, 5 * B + 3
    a, b = (make_pool(L, 4, G, B=B, ns=2, blocks=8, rope=rope) for _ in range(2))
    k, v = randn(1, 1, n, L, G, 128), randn(2, 1, n, L, G, 128)
    order = to_pool_order(rope or Rope(), 128)
    tail = Tail(torch.zeros(1, 3 * B, L, G, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 3 * B, L, G, 128, dtype=torch.bfloat16, device="cuda"), ints([0]))
    ids = [7, 3, 11, 0, 14, 2]
    at, held, done = 0, 0, 0
    steps = [1, 2, B - 3, 5, B, 2 * B - 1] + [1] * (2 * B)
    a.reserve_blocks(1, 2, ids[:2])
    reserved = 2
    for m in steps:
        m = min(m, n - at)
        if m == 0:
            break
        while (held + m + B - 1) // B > a.session_reserved(1):
            a.reserve_blocks(1, 1, [ids[reserved]])
            reserved += 1
        a.append_tokens(k[:, at:at + m], v[:, at:at + m], tail, pages=True, session_first=1)
        tail.n_tokens += m
        at, held = at + m, held + m
        if held >= B:
            a.commit_blocks([held // B], tail, session_first=1)
            done, held = done + held // B, held % B
    assert at == n and done == 5 and a.session_blocks(1) == 5 and int(tail.n_tokens) == held == 3
    raw = k[0, :5 * B][..., order].contiguous()
    b.append_blocks(1, raw, v[0, :5 * B].contiguous(), ids[:5])
    assert torch.equal(a.block_table(1), b.block_table(1)) and torch.equal(a.index(1), b.index(1))
    for p in ids[:5]:
        assert torch.equal(a.pages()[p], b.pages()[p])
    assert torch.equal(tail.v[0, :3], v[0, 5 * B:])                     # what is left of the tail is in front
    assert a.device_status() == 0


def test_a_commit_moves_the_tail_down():
    """Rows behind the committed blocks move to the front, in runs when there are more of them than the blocks held."""
    B, cap = 16, 400
    pool = make_pool(1, 4, 2, B=B, ns=3, blocks=30)
    guards = Guards(dev())
    tail = Tail(guards.empty((3, cap, 1, 2, 128), torch.bfloat16), guards.empty((3, cap, 1, 2, 128), torch.bfloat16), ints([399, 20, 300]))
    tail.k.copy_(randn(1, 3, cap, 1, 2, 128))
    tail.v.copy_(randn(2, 3, cap, 1, 2, 128))
    k0, v0 = tail.k.clone(), tail.v.clone()
    for s in range(3):
        pool.reserve_blocks(s, 20)
    pool.commit_blocks([1, 0, 18], tail)
    torch.cuda.synchronize()
    assert tail.n_tokens.tolist() == [383, 20, 12] and pool.device_status() == 0
    for x, x0 in ((tail.k, k0), (tail.v, v0)):
        assert torch.equal(x[0, :383], x0[0, 16:399]) and torch.equal(x[0, 383:], x0[0, 383:])
        assert torch.equal(x[1], x0[1])
        assert torch.equal(x[2, :12], x0[2, 288:300])
    assert [pool.session_blocks(s) for s in range(3)] == [1, 0, 18] and [pool.session_reserved(s) for s in range(3)] == [19, 20, 2]
    pool.commit_blocks([1, 1, 0], tail)                                 # session 1 has 20 tokens: one block is there
    assert tail.n_tokens.tolist() == [367, 4, 12] and pool.device_status() == 0
    pool.commit_blocks([0, 1, 0], tail)                                 # and no second one
    assert pool.device_status() == kvmem.E_DEVICE_RANGE and tail.n_tokens.tolist() == [367, 0, 12]
    guards.check()


def test_commits_of_many_sessions():
    ns, B = 300, 16
    pool = make_pool(1, 2, 1, B=B, ns=ns, blocks=2, positions=0)
    tail = Tail(randn(1, ns, 40, 1, 1, 128), randn(2, ns, 40, 1, 1, 128), ints([33] * ns))
    for s in range(ns):
        pool.reserve_blocks(s, 2)
    k = randn(3, ns, 32, 1, 1, 128)
    t2 = Tail(tail.k, tail.v, ints([0] * ns))
    pool.append_tokens(k, k, t2, pages=True)
    pool.commit_blocks([s % 3 for s in range(ns)], tail)
    for s in (0, 1, 2, 127, 128, 129, 256, 299):
        assert pool.session_blocks(s) == s % 3 and int(tail.n_tokens[s]) == 33 - 16 * (s % 3)
        if s % 3:
            want = k[s, :16 * (s % 3), 0, 0].float().view(s % 3, 16, 128)
            acc = torch.zeros(s % 3, 128, device="cuda")
            for t in range(16):
                acc = acc + want[:, t]
            assert torch.equal(pool.index(s)[0, 0], (acc * (1.0 / 16)).to(torch.bfloat16))
    assert pool.device_status() == 0


def test_a_captured_append_follows_the_tail():
    c = Append(ns=2, M=3, tails=(4, 60), sel=(3, 1), extra=12)
    c.call()
    torch.cuda.synchronize()
    n_new, n_sel = ints(c.n_new), ints(c.sel)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.pool.append_tokens(c.k, c.v, c.tail, q=c.q, q_out=c.q_out, n_new=n_new, n_sel=n_sel, pages=True)
    for tails, sel in (((4, 60), (3, 1)), ((9, 62), (0, 2)), ((1, 0), (5, 5))):
        c.tails, c.sel = list(tails), list(sel)
        c.tail.n_tokens.copy_(torch.tensor(tails, dtype=torch.int32))
        n_sel.copy_(torch.tensor(sel, dtype=torch.int32))
        for x in (c.tail.k, c.tail.v, c.q_out):
            x.fill_(5.0)
        c.pool.pages().fill_(4.0)
        g.replay()
        c.check()


def test_what_changes_the_hosts_bookkeeping_is_not_captured():
    pool = make_pool(blocks=4)
    tail = Tail(torch.zeros(1, 64, 1, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 64, 1, 2, 128, dtype=torch.bfloat16, device="cuda"), ints([0]))
    pool.reserve_blocks(0, 1)
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    refused = []
    with torch.cuda.graph(g, stream=st):
        tail.n_tokens.add_(0)
        for f in (lambda: pool.reserve_blocks(0, 1), lambda: pool.commit_blocks([1], tail), lambda: pool.set_rope(Rope())):
            try:
                f()
            except KvmemError as e:
                refused.append(e.status)
    assert refused == [kvmem.E_STATE] * 3
    assert pool.session_reserved(0) == 1 and pool.session_blocks(0) == 0


def test_append_and_commit_on_another_stream():
    c = Append(ns=2, M=70, tails=(0,), pages=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c.call()
        st.synchronize()
        c.check()
        c.tail.n_tokens += 70
        c.pool.commit_blocks([1, 1], c.tail)
    st.synchronize()
    assert c.tail.n_tokens.tolist() == [6, 6] and torch.equal(c.tail.v[:, :6], c.v[:, 64:])


def test_what_append_reserve_and_commit_refuse():
    c = Append(ns=2, M=4, tails=(0,), pages=False)
    pool = c.pool
    call = lambda **kw: c.call(**kw)

    def refused(status, f):
        with pytest.raises(KvmemError) as e:
            f()
        assert e.value.status == status, e.value

    refused(kvmem.E_INVALID, lambda: call(first_position=-1))
    refused(kvmem.E_INVALID, lambda: call(first_position=4096))
    refused(kvmem.E_INVALID, lambda: call(q_amplitude=-1.0))
    refused(kvmem.E_INVALID, lambda: call(q_amplitude=math.nan))
    refused(kvmem.E_INVALID, lambda: call(q_out=None))
    refused(kvmem.E_INVALID, lambda: call(q=None))
    refused(kvmem.E_INVALID, lambda: call(pages=True, session_first=1))
    small = Tail(c.tail.k[:, :3].contiguous(), c.tail.v[:, :3].contiguous(), c.tail.n_tokens)
    refused(kvmem.E_INVALID, lambda: pool.append_tokens(c.k, c.v, small))
    refused(kvmem.E_INVALID, lambda: pool.append_tokens(c.k, c.v, Tail(c.tail.k, c.tail.k, c.tail.n_tokens)))        # keys and values in one place
    refused(kvmem.E_INVALID, lambda: pool.append_tokens(c.tail.k[:, :4], c.v, c.tail))                                 # the tail appended to itself
    refused(kvmem.E_INVALID, lambda: call(q=c.q_out))
    for kw in (dict(n_new=ints([1])), dict(n_sel=ints([1, 2]).long()), dict(positions=ints([[1, 2], [3, 4]])), dict(q=c.q.float())):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(ValueError):
        pool.append_tokens(c.k[..., ::2], c.v, c.tail)
    refused(kvmem.E_INVALID, lambda: pool.reserve_blocks(5, 1))
    refused(kvmem.E_INVALID, lambda: pool.reserve_blocks(0, -1))
    refused(kvmem.E_INVALID, lambda: pool.reserve_blocks(0, 1, [99]))
    refused(kvmem.E_INVALID, lambda: pool.reserve_blocks(0, 2, [1, 1]))
    refused(kvmem.E_CAPACITY, lambda: pool.reserve_blocks(0, 3))
    pool.reserve_blocks(0, 0)
    pool.reserve_blocks(0, 1, [1])
    refused(kvmem.E_STATE, lambda: pool.reserve_blocks(1, 1, [1]))
    refused(kvmem.E_STATE, lambda: pool.commit_blocks([2, 0], c.tail))
    refused(kvmem.E_INVALID, lambda: pool.commit_blocks([-1, 0], c.tail))
    refused(kvmem.E_INVALID, lambda: pool.commit_blocks([0, 0], None, session_first=1))
    k = randn(2, 64, 1, 2, 128)
    refused(kvmem.E_STATE, lambda: pool.append_blocks(0, k, k))
    assert pool.session_reserved(0) == 1 and pool.session_reserved(1) == 0
    pool.commit_blocks([0, 0], c.tail)
    pool.session_reset(0)
    assert pool.session_reserved(0) == 0
    pool.append_blocks(0, k, k, [1])                                    # the page is free again
    for other in (Pool(1, 8, 2, 128, 64, 1, 2, 2, dev().index, rope_max_positions=256, rope_theta=THETA, rope_in_block_keys=True),
                  Pool(1, 8, 2, 128, 64, 1, 2, 2, dev().index, fp8_pages=True)):
        refused(kvmem.E_STATE, lambda: other.reserve_blocks(0, 1))
        t = Tail(torch.zeros(1, 8, 1, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 8, 1, 2, 128, dtype=torch.bfloat16, device="cuda"), ints([0]))
        refused(kvmem.E_STATE, lambda: other.append_tokens(c.k[:1], c.v[:1], t, pages=True))
        other.append_tokens(c.k[:1], c.v[:1], t)                        # the tail alone is fine
        assert other.device_status() == 0
    assert bool((c.tail.k == 5.0).all())


# ---- together -------------------------------------------------------------------------------------------------------------------

def test_the_loop_with_a_models_own_rotary_form():
    """Two prompts come in (chunk attention, pages, commits), a question recalls blocks, is prefilled over the view, and is answered
    token by token, with a model of interleaved pairs, a part of the head rotated and scaled frequencies: against the model's own
    arithmetic in 64 bits, keys and queries rounded to bf16 once as they are stored.

    Bounds: those of the attention (2^-8 sum p|v| + 2^-8 |ref|, fp32 sums of n 2^-23), and logits: where the fp32 rotation and the
    64-bit one fall on two sides of a rounding border an element moves by a bf16 step, 2^-7 of it; the two are within 5 * 2^-24 (|a| + |b|),
    so that is one element in some 2^13, and more than four among the 256 of a logit are not met: 4 * 2^-7 max|q| max|k| scale."""
    L, H, G, B, d, ns = 1, 8, 2, 32, 128, 2
    rope = Rope("interleaved", 96, "ramp", 4.0, 512.0)
    pool = make_pool(L, H, G, B=B, ns=ns, blocks=40, positions=2048, rope=rope)
    order = to_pool_order(rope, d)
    n_prompt, n_ask, n_answer = 700, 90, 40
    total = n_prompt + n_ask + n_answer
    q, k, v = randn(1, ns, total, L, H, d), randn(2, ns, total, L, G, d), randn(3, ns, total, L, G, d)
    cap = 1000
    tail = Tail(torch.zeros(ns, cap, L, G, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(ns, cap, L, G, d, dtype=torch.bfloat16, device="cuda"), ints([0] * ns))

    def stored(x, pos):
        return turned(x.double()[..., order], pos.view(-1, 1, 1), rope)[0].to(torch.bfloat16).double()

    def reference(s, rows, pos_q, keys, pos_k, sees):
        """rows, keys: token numbers; [rows][H][d] outputs, sum p|v|, dx"""
        qs = stored(q[s, rows], pos_q)[:, 0]                            # [rows][H][d]
        ks, vs = stored(k[s, keys], pos_k)[:, 0], v[s, keys].double()[:, 0]
        kk, vv = ks.repeat_interleave(H // G, 1), vs.repeat_interleave(H // G, 1)
        x = torch.einsum("ihd,jhd->hij", qs, kk) / math.sqrt(d)
        x = torch.where(sees, x, -math.inf)
        p = torch.softmax(x, 2)
        dx = 4 * 2.0 ** -7 * qs.abs().max().item() * ks.abs().max().item() / math.sqrt(d)
        return torch.einsum("hij,jhd->ihd", p, vv), torch.einsum("hij,jhd->ihd", p, vv.abs()), dx

    def check(out, s, ref):
        want, absv, dx = ref
        got = out.double()
        tol = (2.0 ** -8 + 2.0 ** -10 + 2 * dx) * absv * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max().item()
        # and it is the right attention, not one that the bound happens to hold: mean error far below the mean size
        assert (got - want).abs().mean().item() < 0.02 * want.abs().mean().item()

    empty, zero = pool.new_view(ns, B), ints([0] * ns)
    at = 0
    for m in (300, 1, 399):                                             # the prompt, in three chunks
        rows = slice(at, at + m)
        for s in range(ns):
            need = (int(tail.n_tokens[s]) + m + B - 1) // B - pool.session_reserved(s)
            pool.reserve_blocks(s, max(need, 0))
        q_rot = torch.zeros(ns, m, L, H, d, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.zeros_like(q_rot), torch.zeros(ns, m, L, H, device="cuda")
        pool.append_tokens(k[:, rows], v[:, rows], tail, q=q[:, rows], q_out=q_rot, pages=True)
        pool.view_prefill_attend(q_rot, empty, zero, tail, out, lse)
        tail.n_tokens += m
        for s in range(ns):
            i, j = torch.arange(at, at + m, device="cuda"), torch.arange(at + m, device="cuda")
            check(out[s, :, 0], s, reference(s, i, i, j, j, j.view(1, -1) <= i.view(-1, 1)))
        at += m
    n_blocks = n_prompt // B
    pool.commit_blocks([n_blocks] * ns, tail)
    assert tail.n_tokens.tolist() == [n_prompt - n_blocks * B] * ns
    # the question: its raw queries score the blocks (the pool's order without a turn: position 0)
    ask = slice(n_prompt, n_prompt + n_ask)
    raw = pool.rope_apply(q[:, ask].reshape(ns * n_ask, H, d), torch.zeros(ns * n_ask, dtype=torch.int32, device="cuda")).view(ns, n_ask, L, H, d)
    assert torch.equal(raw, q[:, ask][..., order])
    budget = 6
    sel, n_sel = torch.zeros(ns, budget, dtype=torch.int32, device="cuda"), ints([0] * ns)
    scores = torch.zeros(ns, 40, device="cuda")
    pool.select(raw, SelectParams(budget, 1 << 20, 0, 1, 1), sel, n_sel, scores)
    for s in range(ns):
        kbar = k[s, :n_blocks * B, 0].double().view(n_blocks, B, G, d).mean(1).repeat_interleave(H // G, 1)
        R = torch.softmax(torch.einsum("ihd,bhd->hib", q[s, ask, 0].double(), kbar) / math.sqrt(d), 2).mean(0).sum(0)
        assert bool(((scores[s, :n_blocks].double() - R).abs() <= 5e-3 * R).all())      # (the index holds bf16 means)
    view = pool.new_view(ns, budget * B)
    pool.materialize_rope(sel, n_sel, view)
    # the tail's tokens move behind the view, then the question joins them
    left = n_prompt - n_blocks * B
    keep = slice(n_blocks * B, n_prompt)
    tail.n_tokens.zero_()
    pool.append_tokens(k[:, keep], v[:, keep], tail, n_sel=n_sel)
    tail.n_tokens += left

    def recalled(s):
        return torch.cat([torch.arange(b * B, (b + 1) * B, device="cuda") for b in sel[s, :int(n_sel[s])].tolist()])

    def step(first, m, attend):
        rows = slice(first, first + m)
        for s in range(ns):
            need = (int(tail.n_tokens[s]) + m + B - 1) // B - pool.session_reserved(s)
            pool.reserve_blocks(s, max(need, 0))
        q_rot = torch.zeros(ns, m, L, H, d, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.zeros_like(q_rot), torch.zeros(ns, m, L, H, device="cuda")
        pool.append_tokens(k[:, rows], v[:, rows], tail, q=q[:, rows], q_out=q_rot, n_sel=n_sel, pages=True)
        attend(q_rot, view, n_sel, tail, out, lse)
        for s in range(ns):
            old = recalled(s)
            T = old.numel()
            i = torch.arange(first, first + m, device="cuda")
            keys = torch.cat([old, torch.arange(n_blocks * B, first + m, device="cuda")])
            pos_k = torch.arange(keys.numel(), device="cuda")
            check(out[s, :, 0], s, reference(s, i, T + i - n_blocks * B, keys, pos_k, keys.view(1, -1) <= i.view(-1, 1)))
        tail.n_tokens += m

    # reserved pages already hold the tail's first tokens: they came with the prompt
    step(n_prompt, n_ask, pool.view_prefill_attend)
    for i in range(n_answer):
        step(n_prompt + n_ask + i, 1, pool.view_tree_attend)
    done = (left + n_ask + n_answer) // B
    pool.commit_blocks([done] * ns, tail)
    end = (n_blocks + done) * B
    for s in range(ns):
        assert pool.session_blocks(s) == n_blocks + done
        acc = torch.zeros(n_blocks + done, G, d, device="cuda")
        kk = k[s, :end, 0][..., order].float().view(n_blocks + done, B, G, d)
        for t in range(B):
            acc = acc + kk[:, t]
        assert torch.equal(pool.index(s)[0].transpose(0, 1), (acc * (1.0 / B)).to(torch.bfloat16))
    assert pool.device_status() == 0
