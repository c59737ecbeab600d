"""Rotation and append of so many tokens that a thread takes several vectors (four and three): the other table of sizes beside that of
few tokens, with vector counts that leave a thread with fewer.  Bounds: those of the tests of few tokens."""
import pytest
import torch

from kvmem_harness import Guards
from paper_2609_04852_b200 import Rope
from paper_2609_04852_b200 import kvmem
from test_gpu_tokens import FORMS, Append, close, dev, make_pool, randn, to_pool_order, turned

pytestmark = pytest.mark.gpu
FEW = 148 * 1024                     # threads of a vector each that are resident together: what is more takes the other kernel


def positions(seed, n, window=4096):
    return torch.randint(0, window, (n,), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()


def many(n_vec, d=128, more=37):
    """The fewest rows that the kernel of several vectors takes, and some."""
    return FEW // (n_vec * (d // 16)) + 1 + more


SIZES = [(1, 128), (2, 128), (3, 128), (5, 128), (7, 128), (40, 128), (6, 16), (5, 64), (3, 80), (9, 256), (7, 512)]


@pytest.mark.parametrize("i", range(len(SIZES)))
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_of_many_matches_the_definition(i, inverse):
    n_vec, d = SIZES[i]
    rows = many(n_vec, d)
    for j, (layout, orders) in enumerate(((a, b) for a in ("half", "interleaved") for b in (("model", "pool"), ("pool", "model"), ("model", "model")))):
        rope = Rope(layout, max(16, d // 32 * 16) if j % 2 else 0, ("none", "ramp", "bands")[j % 3], 1.0 if j % 3 == 0 else 4.0, 512.0)
        pool = make_pool(H=1, G=1, d=d, rope=rope)
        x, pos, amplitude = randn(100 * i + j, rows, n_vec, d), positions(i, rows), 1.0 if j % 2 else 1.25
        guards = Guards(dev())
        out = guards.empty((rows, n_vec, d), torch.bfloat16, fill=9.0)
        pool.rope_apply(x, pos, out=out, inverse=inverse, amplitude=amplitude, x_order=orders[0], out_order=orders[1])
        assert pool.device_status() == 0
        order = to_pool_order(rope, d)
        xp = x.double() if orders[0] == "pool" else x.double()[..., order]
        close(out if orders[1] == "pool" else out[..., order], *turned(xp, pos.view(-1, 1), rope, sign=-1.0 if inverse else 1.0, amplitude=amplitude))
        guards.check()
        # the bits of the kernel that takes few
        for lo in range(0, rows, 300):
            if n_vec * (d // 16) * 300 <= FEW:
                part = pool.rope_apply(x[lo:lo + 300], pos[lo:lo + 300], inverse=inverse, amplitude=amplitude, x_order=orders[0], out_order=orders[1])
                assert torch.equal(part, out[lo:lo + 300])
            if lo >= 3000:
                break


@pytest.mark.parametrize("i", range(len(FORMS)))
def test_every_form_of_many(i):
    rope = FORMS[i]
    pool = make_pool(rope=rope)
    rows = many(5)
    x, pos = randn(i, rows, 5, 128), positions(i, rows)
    for inverse in (False, True):
        out = pool.rope_apply(x, pos, inverse=inverse)
        close(out, *turned(x.double()[..., to_pool_order(rope, 128)], pos.view(-1, 1), rope, sign=-1.0 if inverse else 1.0))
    assert pool.device_status() == 0


@pytest.mark.parametrize("n_vec", [5, 40])
def test_strides_of_many(n_vec):
    rope = Rope("interleaved", 64)
    pool = make_pool(rope=rope)
    rows = many(n_vec)
    pos = positions(3, rows)
    wide = randn(1, rows, (n_vec + 7) * 128)
    x = wide[:, 5 * 128:(5 + n_vec) * 128].unflatten(1, (n_vec, 128))
    plain = pool.rope_apply(x.contiguous(), pos)
    assert torch.equal(pool.rope_apply(x, pos), plain)
    heads_first = torch.zeros(n_vec, rows, 128, dtype=torch.bfloat16, device="cuda")
    pool.rope_apply(x, pos, out=heads_first.transpose(0, 1))
    assert torch.equal(heads_first.transpose(0, 1), plain)
    assert torch.equal(pool.rope_apply(heads_first.transpose(0, 1), pos, x_order="pool"), pool.rope_apply(plain, pos, x_order="pool"))
    assert torch.equal(pool.rope_apply(x[:, :1].expand(rows, n_vec, 128), pos), plain[:, :1].expand(rows, n_vec, 128))
    before = wide.clone()
    same = pool.rope_apply(x, pos, out_order="model")
    pool.rope_apply(x, pos, out=x, out_order="model")
    before[:, 5 * 128:(5 + n_vec) * 128] = same.flatten(1)
    assert torch.equal(wide, before)
    assert pool.device_status() == 0


@pytest.mark.parametrize("n_vec", [1, 6, 7])
def test_positions_outside_the_table_among_many(n_vec):
    pool = make_pool(positions=100, rope=Rope("interleaved"))
    rows = many(n_vec)
    pos = positions(1, rows, 100)
    bad = [0, 5, 127, 128, rows // 2, rows - 1]
    for r, p in zip(bad, (-1, 100, 2 ** 31 - 1, -2 ** 31, 101, -7)):
        pos[r] = p
    guards = Guards(dev())
    out = guards.empty((rows, n_vec, 128), torch.bfloat16, fill=7.0)
    pool.rope_apply(randn(1, rows, n_vec, 128), pos, out=out)
    assert pool.device_status() == kvmem.E_DEVICE_RANGE and pool.device_status() == 0
    assert (out == 7.0).flatten(1).all(1).nonzero().flatten().tolist() == bad
    guards.check()


def test_more_rows_than_a_launch_takes():
    """A launch takes 2^30 threads: rows behind that begin another, at rows, vectors and positions of their own."""
    d, heads = 16, 1                                                     # a thread a row: the threads are the rows' number
    rows = (1 << 30) + 12345
    pool = make_pool(H=1, G=1, d=d, positions=512, rope=Rope("interleaved"))
    x = randn(1, 1 << 16, heads, d).repeat(rows // (1 << 16) + 1, 1, 1)[:rows]
    pos = positions(2, 1 << 16, 512).repeat(rows // (1 << 16) + 1)[:rows]
    pool.rope_apply(x, pos, out=x, out_order="model")
    want = pool.rope_apply(randn(1, 1 << 16, heads, d), pos[:1 << 16], out_order="model")
    for lo in (0, 1 << 16, (1 << 30) - (1 << 16), 1 << 30):
        n = min(1 << 16, rows - lo)
        assert torch.equal(x[lo:lo + n], want[:n])
    assert pool.device_status() == 0
    del x, pos
    torch.cuda.empty_cache()


APPENDS = [
    dict(M=2800, H=5, G=1, rope=Rope("interleaved", 96, "ramp", 8.0, 512.0)),                  # 7 vectors: one left over
    dict(M=1700, H=4, G=1, L=2, tails=(100,), rope=Rope("half", 64)),                     # 12
    dict(M=2700, H=6, G=1, tails=(0,), B=16),                                                  # 8: two left over
    dict(ns=3, M=1000, n_new=(1000, 0, 777), H=5, G=1, tails=(5, 0, 130), sel=(1, 0, 9), first=100, amplitude=1.75, rope=Rope("interleaved", 32)),
    dict(ns=2, M=700, n_new=(699, 700), L=2, H=4, G=2, tails=(63, 1), explicit=True, amplitude=1.5, rope=Rope("interleaved", 0, "bands", 8.0, 300.0)),
    dict(M=2500, H=4, G=4, queries=False, rope=Rope("interleaved")),                           # keys and values alone: 8
    dict(M=1700, H=6, G=2, L=3, pages=False, tails=(900,), amplitude=1.75, rope=Rope("half", 16, "linear", 4.0)),
    dict(ns=2, M=900, H=9, G=1, B=16, packed=False, tails=(2, 9), rope=Rope("interleaved")),   # 11
    dict(M=2800, H=5, G=1, positions=0, sel=None),                                             # copies
    dict(M=1400, H=5, G=1, d=256, sel=None, rope=Rope("half", 64, "base", 2.0)),
    dict(M=3100, H=6, G=2, d=80, B=48, sel=None, amplitude=0.75, rope=Rope("interleaved", 48)),
    dict(ns=70, M=40, n_new=[(7 * s) % 41 for s in range(70)], H=5, G=1, tails=(0, 3, 64, 17), sel=(3, 0), B=32, rope=Rope("interleaved", 64)),
]


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append_of_many_matches_the_definition(i):
    c = Append(seed=50 + i, **APPENDS[i])
    vectors = c.L * ((c.H if c.q is not None else 0) + 2 * c.G)
    assert c.ns * c.M > FEW // (vectors * (c.d // 16))
    c.call()
    c.check()
    c.call()
    c.check()


def test_positions_and_lengths_out_of_range_among_many():
    c = Append(M=2800, H=5, G=1, tails=(3,), positions=4096, sel=(2,), first=60, pages=False)
    c.call(first_position=4096 - 128 - 3 - 2000)                         # row 3 + i at 4096 - 2000 + i
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE
    for x in (c.tail.k[:, 3:], c.tail.v[:, 3:], c.q_out):
        assert bool((x[:, 2000:] == 5.0).all()) and not bool((x[:, :2000] == 5.0).flatten(2).all(-1).any())
    c.guards.check()
    c = Append(M=2800, H=5, G=1, tails=(9,), extra=0, pages=False)
    c.tail.n_tokens.fill_(2 ** 31 - 1)
    c.call()
    c.tail.n_tokens.fill_(9)
    c.check(status=kvmem.E_DEVICE_RANGE)


def test_rows_without_a_page_among_many():
    c = Append(M=2800, H=5, G=1, tails=(0,), sel=None, pages=False)
    c.pool.reserve_blocks(0, 2, [5, 1])
    c.call(pages=True)
    torch.cuda.synchronize()
    assert c.pool.device_status() == kvmem.E_DEVICE_RANGE and torch.equal(c.tail.v[:, :2800], c.v)
    for p in range(c.pool.pages().shape[0]):
        b = {5: 0, 1: 1}.get(p)
        got = c.pool.pages()[p, 1, 0]
        assert bool((got == 4.0).all()) if b is None else torch.equal(got, c.v[0, 64 * b:64 * b + 64, 0].transpose(0, 1))
    c.guards.check()
