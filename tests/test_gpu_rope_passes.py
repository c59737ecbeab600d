"""The passes that rotate, on a pool with a model's own rotary form, against attention in 64 bits over the definition's keys: raw keys
turned to their compact positions without a rounding.

Bounds.  What separates a pass from the definition are roundings to bf16: of a turned key (once on a raw pool; a block of the execution
cache that moved is turned and rounded once more; a key rotated in its block is stored rounded and turned again), of the query that the
copy-free pass of an in-block pool turns back to each block, and of the weights.  Each is off by at most 2^-8 of the element (of its pair's length, where
it is turned afterwards), either way.  To first order the error of an output is a sum of them with fixed factors c,
    of a key's element i at token t:  p_t (v_t - out) scale q_i 2^-8 k_ti      of a weight:  2^-8 p_t v_t
    of a turned query's element at block b:  2^-8 q_i scale sum over t in b of p_t (v_t - out) k_ti
and of the log-sum-exp the same without (v - out).  For independent errors of mean 0 Hoeffding's inequality gives
P(|sum| >= z sqrt(sum c^2)) <= 2 exp(-z^2 / 2): below 10^-12 for z = 7.6, some 10^6 values being compared.  Second order: the logits move by less than
2^-6 altogether, so at most 2^-6 of the first.  fp32 sums: 320 tokens and 128 products, 10^-5 on values of unit scale."""
import math

import pytest
import torch

from kvmem_harness import ATTN_ATOL
from test_gpu_tokens import FORMS, ints, make_pool, randn, turned

pytestmark = pytest.mark.gpu
D, Z = 128, 7.6


def lengths(x):
    """Of the pairs (i, i + d/2), at both their places."""
    n = (x[..., :D // 2] ** 2 + x[..., D // 2:] ** 2).sqrt()
    return torch.cat([n, n], -1)


class Definition:
    """Query head by query head, q fp64 [M][H][d] and k, v fp64 [T][G][d]."""

    def __init__(self, q, k, v, B):
        M, H, _ = q.shape
        T, G, _ = k.shape
        scale = 1.0 / math.sqrt(D)
        qq, r = q.view(M, G, H // G, D), H // G
        p = torch.softmax(torch.einsum("mgrd,tgd->mgrt", qq, k) * scale, -1)
        self.out = torch.einsum("mgrt,tgd->mgrd", p, v)
        self.lse = torch.logsumexp(torch.einsum("mgrd,tgd->mgrt", qq, k) * scale, -1)
        away = (v.permute(1, 0, 2).view(1, G, 1, T, D) - self.out.unsqueeze(3)) * p.unsqueeze(-1)         # [m][g][r][t][d]
        step = scale * 2.0 ** -8
        kq = torch.einsum("mgrd,tgd->mgrt", lengths(qq) ** 2, lengths(k) ** 2) / 2                        # (a pair is there twice)
        self.key_out = torch.einsum("mgrt,mgrtd->mgrd", kq, away ** 2) * step ** 2
        self.key_lse = (kq * p ** 2).sum(-1) * step ** 2
        self.weight = torch.einsum("mgrt,tgd->mgrd", p ** 2, v ** 2) * 2.0 ** -16
        # by blocks, elements of the pair's length: sum over i of |q_i|^2 |sum over t of p (v - out) k_ti|^2
        ab = torch.einsum("mgrbtd,btge->mgrbde", away.view(M, G, r, T // B, B, D), k.view(T // B, B, G, D))
        self.query_out = torch.einsum("mgre,mgrbde->mgrd", lengths(qq) ** 2, ab ** 2) * step ** 2
        pb = torch.einsum("mgrbt,btge->mgrbe", p.view(M, G, r, T // B, B), k.view(T // B, B, G, D))
        self.query_lse = torch.einsum("mgre,mgrbe->mgr", lengths(qq) ** 2, pb ** 2) * step ** 2

    def check(self, out, lse, keys, queries):
        got, gl = out.double().view(self.out.shape), lse.double().view(self.lse.shape)
        tol = Z * (keys * self.key_out + queries * self.query_out + self.weight).sqrt() * (1 + 2.0 ** -6) + 1e-5
        ltol = Z * (keys * self.key_lse + queries * self.query_lse).sqrt() * (1 + 2.0 ** -6) + 1e-5
        err, lerr = (got - self.out).abs(), (gl - self.lse).abs()
        assert bool((err <= tol).all()), (err / tol).max().item()
        assert bool((lerr <= ltol).all()), (lerr / ltol).max().item()
        assert err.mean().item() < 0.01 * self.out.abs().mean().item()
        return err.max().item(), lerr.max().item()


@pytest.mark.parametrize("in_block", [False, True])
@pytest.mark.parametrize("i", range(len(FORMS)))
def test_attention_of_every_pass_is_that_of_the_definition(i, in_block):
    rope, B, NB, G, H, M, first = FORMS[i], 64, 12, 2, 8, 3, 100
    pool = make_pool(1, H, G, B=B, blocks=NB, positions=2048, rope=rope, rope_in_block_keys=in_block)
    raw, v = randn(i, NB * B, 1, G, D), randn(50 + i, NB * B, 1, G, D)
    pool.append_blocks(0, raw, v)
    ids = [0, 3, 4, 9, 11]
    sel, n_sel = ints([ids]), ints([len(ids)])
    tok = torch.cat([torch.arange(b * B, (b + 1) * B) for b in ids]).cuda()
    where = first + torch.arange(tok.numel(), device="cuda")
    q = pool.rope_apply(randn(90 + i, M, H, D), ints([first + tok.numel()] * M)).view(1, M, 1, H, D)
    want = Definition(q.double().view(M, H, D), turned(raw[tok, 0].double(), where.view(-1, 1), rope)[0], v[tok, 0].double(), B)
    keys = 2 if in_block else 1
    worst = []

    def check(out, lse, keys, queries=0):
        worst.append(max(want.check(out, lse, keys, queries)))

    views = [pool.new_view(1, len(ids) * B) for _ in range(2)]
    outs = [pool.new_outputs(1, M) for _ in range(3)]
    pool.materialize_rope(sel, n_sel, views[0], first)
    pool.view_attend(q, views[0], n_sel, *outs[0])
    check(*outs[0], keys)
    pool.paged_attend_rope(q, sel, n_sel, *outs[1], first_position=first)
    check(*outs[1], 1, 1 if in_block else 0)
    pool.materialize_attend_rope(q, sel, n_sel, views[1], *outs[2], first_position=first)
    check(*outs[2], keys)
    if not in_block:
        cache = pool.new_view_cache(len(ids), 2, first)
        cache.update(0, ints([0, 1, 2, 9, 11]), n_sel)
        cache.update(0, sel[0].contiguous(), n_sel)                     # two blocks stay and turn on by a difference
        out, lse = pool.new_outputs(1, M)
        cache.attend(q[0], out[0], lse[0])
        check(out, lse, 2)
        assert max(worst) <= ATTN_ATOL                                  # what the other passes' tests ask of unit-scale values
    assert pool.device_status() == 0
