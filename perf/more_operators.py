"""Measured cases of what brings new tokens into the cache: what each computes, on which sizes, and what it must move.

  rope     queries or keys rotated to their positions in the model's own form (halves or interleaved pairs, a part of the
           head, frequencies scaled for long contexts), or back (``Pool.set_rope``, ``Pool.rope_apply``)
  append   new tokens' queries, keys and values out of a packed projection: rotated queries, rotated keys and values behind
           the tail's committed tokens, raw keys and values in the reserved pages (``Pool.reserve_blocks``,
           ``Pool.append_tokens``)
  prefill  attention of a prompt chunk over the execution view, the committed tail and the chunk itself
           (``Pool.view_prefill_attend``)

``run`` computes them in elementary torch operations in 32 bits (angles in 64); with ``own`` set it calls the package
instead.  ``exact`` computes them once more, in 64 bits, written apart.

A head's dims in the pool's order: pair i of the rotation at i and d/2 + i, the dims that do not rotate behind the pairs of
either half.  Any rotary form is this one after a fixed permutation of the dims, which no product of a query and a key sees.
"""
from __future__ import annotations

import math

import torch

own = False

THETA = 1.0e6                # rotary base of this repository's benchmark


# ------------------------------------------------------------------------------------------------ cases

def _rope(name, rows, heads, dim, layout, rotary, scaling, factor, window, inverse, packed, order, amplitude):
    return {"name": name, "op": "rope", "rows": rows, "heads": heads, "dim": dim, "layout": layout, "rotary": rotary,
            "scaling": scaling, "factor": factor, "window": window, "inverse": inverse, "packed": packed, "order": order,
            "amplitude": amplitude}


def _append(name, sessions, layers, heads, kv_heads, block, new, tail, ragged, pages, layout, rotary, scaling, factor, window):
    return {"name": name, "op": "append", "sessions": sessions, "layers": layers, "heads": heads, "kv_heads": kv_heads, "dim": 128,
            "block": block, "new": new, "tail": tail, "ragged": ragged, "pages": pages, "layout": layout, "rotary": rotary,
            "scaling": scaling, "factor": factor, "window": window}


def _prefill(name, sessions, layers, heads, kv_heads, block, blocks, new, tail, ragged):
    return {"name": name, "op": "prefill", "sessions": sessions, "layers": layers, "heads": heads, "kv_heads": kv_heads, "dim": 128,
            "block": block, "blocks": blocks, "new": new, "tail": tail, "ragged": ragged}


def listed():
    return [
        # one decode step of eight sessions, 32 query and 8 key heads each, far positions: latency counts
        _rope("rope 8 x 40, interleaved", 8, 40, 128, "interleaved", 128, "none", 1.0, 131072, False, False, "pool", 1.0),
        # the queries and keys of a 2,048-token prompt chunk as they lie in the packed projection, half of the head rotated,
        # scaled frequencies with the amplitude that goes with them
        _rope("rope 2k x 40 packed, ramp", 2048, 40, 128, "half", 64, "ramp", 4.0, 131072, False, True, "pool", 1.2965),
        # cached keys of 32,777 tokens brought back to raw form
        _rope("rope 32k x 8 back, bands", 32777, 8, 128, "half", 128, "bands", 8.0, 262144, True, False, "model", 1.0),
        # a whole prompt in the model's own order, longer than any cache
        _rope("rope 24k x 40, linear", 24576, 40, 128, "interleaved", 96, "linear", 2.0, 32768, False, False, "model", 1.0),
        # one decoded token of eight sessions, with its page rows
        _append("append 8 x 1", 8, 1, 32, 8, 64, 1, 41, False, True, "half", 128, "none", 1.0, 262144),
        # drafted tokens of eight sessions, padded, two layers, 32-token blocks; the tail alone
        _append("append 8 x 12 ragged drafts", 8, 2, 16, 4, 32, 12, 90, True, False, "interleaved", 64, "base", 4.0, 65536),
        # a prompt chunk, with its page rows
        _append("append chunk 2k", 1, 1, 32, 8, 64, 2048, 63, False, True, "half", 128, "ramp", 4.0, 131072),
        # a long prompt at once, odd length and start, with its page rows
        _append("append prompt 16k", 1, 1, 32, 8, 64, 16383, 19, False, True, "interleaved", 128, "none", 1.0, 32768),
        # a short question over the view of the 16,384-token history
        _prefill("prefill 129 over 2k", 1, 1, 32, 8, 64, 32, 129, 37, False),
        # a fresh prompt of 4,096 tokens, nothing recalled: the causal part alone
        _prefill("prefill 4k fresh", 1, 1, 32, 8, 64, 0, 4096, 0, False),
        # three sessions of different lengths, two layers, five query heads on a KV head, padded chunks
        _prefill("prefill batch 3 ragged, 700", 3, 2, 20, 4, 32, 301, 700, 115, True),
        # the paper's 2,048-token chunk over its 64K view
        _prefill("prefill 2k over 64k", 1, 1, 32, 8, 64, 1024, 2048, 50, False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "append", "prefill"))
    layout, scaling = rng.choice(("half", "interleaved")), rng.choice(("none", "linear", "base", "ramp", "bands"))
    factor = 1.0 if scaling == "none" else float(rng.choice((2, 4, 8)))
    if op == "rope":
        dim = rng.choice((64, 128, 128, 128, 256))
        heads = rng.choice((1, 2, 5, 8, 12, 32, 40))
        rows = _log(rng, 1, min(100000, 24576 * 40 * 128 // (heads * dim)))
        return _rope("", rows, heads, dim, layout, 16 * rng.randint(1, dim // 16), scaling, factor, _log(rng, 1024, 262144),
                     rng.random() < 0.4, rng.random() < 0.4, rng.choice(("pool", "model")), rng.choice((1.0, 1.0, 1.2079)))
    sessions, layers = _log(rng, 1, 8), rng.choice((1, 1, 2, 3))
    kv_heads, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 4, 5, 8))
    block = rng.choice((16, 32, 64, 64, 128))
    ragged = sessions > 1 and rng.random() < 0.7
    tail = rng.choice((0, _log(rng, 1, 300)))
    if op == "append":
        new = _log(rng, 1, max(2, 16000 * 48 // (sessions * layers * kv_heads * (group + 2))))
        new = min(new, 20000)
        return _append("", sessions, layers, kv_heads * group, kv_heads, block, new, tail, ragged, rng.random() < 0.6, layout,
                       16 * rng.randint(1, 8), scaling, factor, 32768 * rng.choice((1, 2, 4)))
    # at most the pairs of the largest case: 32 heads x 2,048 tokens x 65,536 tokens
    pairs = 32 * 2048 * 65536 // (sessions * layers * kv_heads * group)
    new = _log(rng, 65, max(66, min(4096, int(math.sqrt(pairs) / 2))))
    blocks = rng.choice((0, _log(rng, 1, max(2, min(4096, (pairs // new - tail - new) // block))),
                         _log(rng, 1, max(2, min(4096, (pairs // new - tail - new) // block)))))
    return _prefill("", sessions, layers, kv_heads * group, kv_heads, block, blocks, new, tail, ragged)


# ------------------------------------------------------------------------------------------------ inputs

def _blocks_of(case):
    """Blocks in each session's view: equal, or from none to all of them in a fixed ragged pattern."""
    n, k = case["sessions"], case["blocks"]
    if not case["ragged"]:
        return [k] * n
    return [k if s == 0 else 0 if s == n - 1 and n > 2 else (k * (2 * s + 3)) // (2 * n + 3) for s in range(n)]


def _new_of(case):
    """New tokens of each session: a padded batch where the case is ragged."""
    n, m = case["sessions"], case["new"]
    return [m if s == 0 or not case["ragged"] else max(1, m - (m * (3 * s % 7)) // 9) for s in range(n)]


def _tails_of(case):
    n, t = case["sessions"], case["tail"]
    return [t if s == 0 or not case["ragged"] else (t * (s + 1)) // (n + 1) for s in range(n)]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _packed(gen, rows, width, extra):
    """[rows][width] as a slice of a wider projection's output."""
    return _normal(gen, rows, width + extra).to(torch.bfloat16)[:, :width]


def _original(case):
    """Window that the scaled frequencies were made for."""
    return max(256, int(case["window"] / case["factor"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    dev, d = "cuda", case["dim"]
    st = {"case": dict(case)}
    if case["op"] == "rope":
        rows, heads = case["rows"], case["heads"]
        st["x"] = (_packed(gen, rows, heads * d, 8 * d) if case["packed"] else _normal(gen, rows, heads * d).to(torch.bfloat16))
        st["x"] = st["x"].unflatten(1, (heads, d))
        st["positions"] = torch.randint(0, case["window"], (rows,), generator=gen, device=dev, dtype=torch.int32)
        st["out"] = torch.zeros(rows, heads, d, dtype=torch.bfloat16, device=dev)
        if own:
            st["pool"] = _pool(case, 1, 1, 1, 64, 1, 1)
        return st
    S, L, H, G, B, M = (case[x] for x in ("sessions", "layers", "heads", "kv_heads", "block", "new"))
    cap = case["tail"] + M + (B if case["op"] == "append" else 0)
    st["n_tail"] = torch.tensor(_tails_of(case), dtype=torch.int32, device=dev)
    st["n_new"] = torch.tensor(_new_of(case), dtype=torch.int32, device=dev)
    if case["op"] == "append":
        # one projection's rows: [L][query, key, value heads][d]
        x = _normal(gen, S, M, L, H + 2 * G, d).to(torch.bfloat16)
        st["q"], st["k"], st["v"] = x[..., :H, :], x[..., H:H + G, :], x[..., H + G:, :]
        st["n_sel"] = torch.randint(0, max(1, (case["window"] - cap) // B), (S,), generator=gen, device=dev, dtype=torch.int32)
        st["q_out"] = torch.zeros(S, M, L, H, d, dtype=torch.bfloat16, device=dev)
        st["tail_k"] = _normal(gen, S, cap, L, G, d).to(torch.bfloat16)
        st["tail_v"] = _normal(gen, S, cap, L, G, d).to(torch.bfloat16)
        per = (cap + B - 1) // B
        perm = torch.randperm(S * per, generator=torch.Generator().manual_seed(int(seed))).view(S, per)
        st["table"] = perm.to(dev)
        if not own:
            st["pages"] = torch.zeros(S * per, 2, L, G, B, d, dtype=torch.bfloat16, device=dev) if case["pages"] else None
        else:
            from paper_2609_04852_b200 import Tail
            st["pool"] = _pool(case, L, H, G, B, S, per)
            st["tail"] = Tail(st["tail_k"], st["tail_v"], st["n_tail"])
            st["pages"] = st["pool"].pages() if case["pages"] else None
            if case["pages"]:
                st["pages"].zero_()
                for s in range(S):
                    st["pool"].reserve_blocks(s, per, perm[s].tolist())
        return st
    cap_view = max(case["blocks"], 1) * B
    u = _normal(gen, S, L * G, d)
    u /= u.norm(dim=-1, keepdim=True)
    q = _normal(gen, S, M, L, G, H // G, d) + math.sqrt(d) * u.view(S, 1, L, G, 1, d)
    st["q"] = q.view(S, M, L, H, d).to(torch.bfloat16)
    k = _normal(gen, S, L * G, cap_view, d)
    planted = torch.rand(S, 1, cap_view // B, generator=gen, device=dev) < 1.0 / 16
    k += 3.0 * planted.repeat_interleave(B, 2).unsqueeze(-1) * u.unsqueeze(2)
    st["k"] = k.to(torch.bfloat16).view(S, L, G, cap_view, d)
    st["v"] = _normal(gen, S, L, G, cap_view, d).to(torch.bfloat16)
    st["n_sel"] = torch.tensor(_blocks_of(case), dtype=torch.int32, device=dev)
    st["tail_k"] = _normal(gen, S, cap, L, G, d).to(torch.bfloat16)
    st["tail_v"] = _normal(gen, S, cap, L, G, d).to(torch.bfloat16)
    st["out"] = torch.zeros(S, M, L, H, d, dtype=torch.bfloat16, device=dev)
    st["lse"] = torch.zeros(S, M, L, H, device=dev)
    if own:
        from paper_2609_04852_b200 import Pool, Tail, View
        st["pool"] = Pool(L, H, G, d, B, S, 1, 1, torch.cuda.current_device())
        st["view"] = View(st["k"], st["v"], cap_view)
        st["tail"] = Tail(st["tail_k"], st["tail_v"], st["n_tail"])
    return st


def _pool(case, layers, heads, kv_heads, block, sessions, blocks):
    from paper_2609_04852_b200 import Pool, Rope
    pool = Pool(layers, heads, kv_heads, case["dim"], block, sessions, sessions * blocks, blocks, torch.cuda.current_device(),
                rope_max_positions=case["window"], rope_theta=THETA)
    pool.set_rope(Rope(case["layout"], case["rotary"], case["scaling"], case["factor"], _original(case)))
    return pool


# ------------------------------------------------------------------------------------------------ plain forms

FAST, SLOW = 32.0, 1.0       # ramp: turns over the original window above / below which a frequency is kept / divided
HIGH, LOW = 4.0, 1.0         # bands: the same, in turns, with a straight line between them


def _frequencies(case):
    """fp64 [rotary / 2]: radians a position adds to each pair's angle."""
    n, factor, window = case["rotary"], case["factor"], _original(case)
    i = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    f = THETA ** (-2.0 * i / n)
    if case["scaling"] == "linear":
        return f / factor
    if case["scaling"] == "base":
        return (THETA * factor ** (n / (n - 2.0))) ** (-2.0 * i / n)
    if case["scaling"] == "ramp":
        lo = max(math.floor(n * math.log(window / (FAST * 2 * math.pi)) / (2 * math.log(THETA))), 0)
        hi = min(math.ceil(n * math.log(window / (SLOW * 2 * math.pi)) / (2 * math.log(THETA))), n - 1)
        divided = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / factor * divided + f * (1 - divided)
    if case["scaling"] == "bands":
        kept = ((window * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return f / factor * (1 - kept) + f * kept
    return f


def _cos_sin(case, positions):
    angle = positions.double().unsqueeze(-1) * _frequencies(case)
    return angle.cos().float(), angle.sin().float()


def _split(x, case, order):
    """fp32 (first, second) elements of the pairs, and the dims that pass."""
    n, d = case["rotary"], case["dim"]
    x = x.float()
    if order == "pool":
        h = d // 2
        return x[..., :n // 2], x[..., h:h + n // 2], torch.cat([x[..., n // 2:h], x[..., h + n // 2:]], -1)
    if case["layout"] == "half":
        return x[..., :n // 2], x[..., n // 2:n], x[..., n:]
    return x[..., 0:n:2], x[..., 1:n:2], x[..., n:]


def _join(a, b, rest, case, order):
    half = rest.shape[-1] // 2
    if order == "pool":
        return torch.cat([a, rest[..., :half], b, rest[..., half:]], -1).to(torch.bfloat16)
    if case["layout"] == "half":
        return torch.cat([a, b, rest], -1).to(torch.bfloat16)
    return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1).to(torch.bfloat16)


def _rotated(x, cos, sin, case, source, target, amplitude=1.0):
    a, b, rest = _split(x, case, source)
    return _join((a * cos - b * sin) * amplitude, (b * cos + a * sin) * amplitude, rest, case, target)


def _orders(case):
    """Order of the dims that come in and that go out: the way back starts from the pool's."""
    return (case["order"], "model") if case["inverse"] else ("model", case["order"])


def _plain_rope(st):
    c = st["case"]
    cos, sin = (t.unsqueeze(1) for t in _cos_sin(c, st["positions"]))
    return _rotated(st["x"], cos, -sin if c["inverse"] else sin, c, *_orders(c), c["amplitude"])


def _plain_append(st):
    c = st["case"]
    S, L, G, B, M, d = (c[x] for x in ("sessions", "layers", "kv_heads", "block", "new", "dim"))
    i = torch.arange(M, device="cuda")
    row = st["n_tail"].long().view(S, 1) + i                                  # [S][M]: row of the tail
    there = (i < st["n_new"].view(S, 1)).view(S, M, 1, 1, 1)
    cos, sin = (t.view(S, M, 1, 1, -1) for t in _cos_sin(c, row + st["n_sel"].long().view(S, 1) * B))
    q = torch.where(there, _rotated(st["q"], cos, sin, c, "model", "pool"), st["q_out"])
    k = _rotated(st["k"], cos, sin, c, "model", "pool")
    at = (torch.arange(S, device="cuda").view(S, 1).expand(S, M), row)
    st["tail_k"][at] = torch.where(there, k, st["tail_k"][at])
    st["tail_v"][at] = torch.where(there, st["v"], st["tail_v"][at])
    if not c["pages"]:
        return q, st["tail_k"], st["tail_v"]
    raw = _join(*_split(st["k"], c, "model"), c, "pool")
    page, place = st["table"].gather(1, row // B), row % B
    for kv, x in ((0, raw), (1, st["v"])):
        to = st["pages"][:, kv].permute(0, 3, 1, 2, 4)                        # [page][token][L][G][d]
        to[page, place] = torch.where(there, x, to[page, place])
    return q, st["tail_k"], st["tail_v"], st["pages"]


def _plain_prefill(st):
    c = st["case"]
    S, L, H, G, M, B, d = (c[x] for x in ("sessions", "layers", "heads", "kv_heads", "new", "block", "dim"))
    r, T = H // G, st["k"].shape[3]
    q = st["q"].float().view(S, M, L, G, r, d).permute(0, 2, 3, 1, 4, 5).reshape(S, L * G, M * r, d)
    q *= 1.0 / math.sqrt(d)
    cap = st["tail_k"].shape[1]
    j = torch.arange(T + cap, device="cuda")
    live = j < (st["n_sel"] * B).view(S, 1)                                   # [S][T + cap]: tokens of the view
    drafted = j - T - st["n_tail"].view(S, 1)                                 # index among the chunk's tokens, negative in front of them
    live = torch.where(j < T, live, drafted < st["n_new"].view(S, 1))
    i = torch.arange(M, device="cuda").view(1, M, 1)
    sees = live.unsqueeze(1) & ((j < T) | (drafted.unsqueeze(1) <= i))        # [S][M][T + cap]
    k, v = (torch.cat([x.flatten(1, 2).float(), t.permute(0, 2, 3, 1, 4).flatten(1, 2).float()], 2)
            for x, t in ((st["k"], st["tail_k"]), (st["v"], st["tail_v"])))
    x = torch.matmul(q, k.transpose(2, 3))
    x.view(S, L * G, M, r, T + cap).masked_fill_(~sees.view(S, 1, M, 1, T + cap), -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    x -= top
    x.exp_()
    z = x.sum(3, keepdim=True)
    o = torch.matmul(x, torch.where(live.view(S, 1, T + cap, 1), v, torch.zeros((), device="cuda")))
    o /= torch.where(z > 0, z, torch.ones_like(z))
    lse = top + z.log()
    here = (torch.arange(M, device="cuda") < st["n_new"].view(S, 1)).view(S, M, 1, 1)
    o = o.view(S, L, G, M, r, d).permute(0, 3, 1, 2, 4, 5).reshape(S, M, L, H, d)
    lse = lse.view(S, L, G, M, r).permute(0, 3, 1, 2, 4).reshape(S, M, L, H)
    return torch.where(here.unsqueeze(4), o.to(torch.bfloat16), st["out"]), torch.where(here, lse, st["lse"])


# ------------------------------------------------------------------------------------------------ one pass

def run(st):
    c = st["case"]
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "prefill": _plain_prefill}[c["op"]](st)
    pool = st["pool"]
    if c["op"] == "rope":
        source, target = _orders(c)
        return pool.rope_apply(st["x"], st["positions"], out=st["out"], inverse=c["inverse"], amplitude=c["amplitude"],
                               x_order=source, out_order=target)
    if c["op"] == "append":
        pool.append_tokens(st["k"], st["v"], st["tail"], q=st["q"], q_out=st["q_out"], n_new=st["n_new"], n_sel=st["n_sel"],
                           pages=c["pages"])
        return (st["q_out"], st["tail_k"], st["tail_v"]) + ((st["pages"],) if c["pages"] else ())
    pool.view_prefill_attend(st["q"], st["view"], st["n_sel"], st["tail"], st["out"], st["lse"], n_q=st["n_new"])
    return st["out"], st["lse"]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    d = case["dim"]
    if case["op"] == "rope":
        pairs = case["rows"] * case["heads"] * case["rotary"] // 2
        return {"bytes": case["rows"] * (case["heads"] * d * 4 + 4), "flops": 6 * pairs}
    S, L, H, G = (case[x] for x in ("sessions", "layers", "heads", "kv_heads"))
    new = _new_of(case)
    if case["op"] == "append":
        # q, k and v read once; rotated q, rotated k and v in the tail and, with pages, raw k and v written once
        per = L * d * 2 * (2 * H + 4 * G + (2 * G if case["pages"] else 0))
        return {"bytes": sum(new) * per + 12 * S, "flops": 3 * sum(new) * L * (H + G) * case["rotary"]}
    seen = sum(n * case["block"] + t + m for n, t, m in zip(_blocks_of(case), _tails_of(case), new))
    pairs = sum((n * case["block"] + t) * m + m * (m + 1) // 2 for n, t, m in zip(_blocks_of(case), _tails_of(case), new))
    return {"bytes": L * G * seen * 2 * d * 2 + sum(new) * L * H * (d * 4 + 4) + 12 * S, "flops": 4 * d * L * H * pairs}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_frequency(case, i):
    """Of pair i, in Python's own floating point."""
    n, factor, window = case["rotary"], case["factor"], _original(case)
    f = THETA ** (-2.0 * i / n)
    turns = window * f / (2 * math.pi)
    kind = case["scaling"]
    if kind == "linear":
        return f / factor
    if kind == "base":
        return (THETA * factor ** (n / (n - 2.0))) ** (-2.0 * i / n)
    if kind == "ramp":
        def pair_of(t):       # the (fractional) pair that makes t turns over the original window
            return n * math.log(window / (t * 2 * math.pi)) / (2 * math.log(THETA))
        lo, hi = max(math.floor(pair_of(FAST)), 0), min(math.ceil(pair_of(SLOW)), n - 1)
        share = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
        return f * (1 - share) + f / factor * share
    if kind == "bands":
        share = min(max((turns - LOW) / (HIGH - LOW), 0.0), 1.0)
        return f * share + f / factor * (1 - share)
    return f


def _exact_places(case):
    """(place of pair i's first element, of its second, places that pass) in the model's order, and the same in the pool's."""
    n, d = case["rotary"], case["dim"]
    if case["layout"] == "half":
        model = [(i, n // 2 + i) for i in range(n // 2)]
    else:
        model = [(2 * i, 2 * i + 1) for i in range(n // 2)]
    passing = list(range(n, d))
    pool = [(i, d // 2 + i) for i in range(n // 2)]
    rest = (d - n) // 2
    pool_passing = [n // 2 + i for i in range(rest)] + [d // 2 + n // 2 + i for i in range(rest)]
    return {"model": (model, passing), "pool": (pool, pool_passing)}


def _exact_turn(case, x, positions, sign, source, target, amplitude):
    """x fp64 [..., d], positions fp64 broadcastable to x's leading dims: pair by pair."""
    places = _exact_places(case)
    y = torch.zeros_like(x)
    for i, ((a, b), (ya, yb)) in enumerate(zip(places[source][0], places[target][0])):
        angle = positions * _exact_frequency(case, i)
        c, s = angle.cos(), sign * angle.sin()
        y[..., ya] = amplitude * (x[..., a] * c - x[..., b] * s)
        y[..., yb] = amplitude * (x[..., b] * c + x[..., a] * s)
    y[..., places[target][1]] = x[..., places[source][1]]
    return y


def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    if case["op"] == "rope":
        return _exact_turn(case, st["x"].double(), st["positions"].double().unsqueeze(1), -1.0 if case["inverse"] else 1.0,
                           *_orders(case), case["amplitude"])
    S, L, H, G, B = (case[x] for x in ("sessions", "layers", "heads", "kv_heads", "block"))
    if case["op"] == "append":
        q, tk, tv = st["q_out"].double(), st["tail_k"].double(), st["tail_v"].double()
        pages = st["pages"].double() if case["pages"] else None
        for s in range(S):
            n, n0 = int(st["n_new"][s]), int(st["n_tail"][s])
            at = (int(st["n_sel"][s]) * B + n0 + torch.arange(n, device="cuda")).double().view(n, 1, 1)
            q[s, :n] = _exact_turn(case, st["q"][s, :n].double(), at, 1.0, "model", "pool", 1.0)
            k, v = st["k"][s, :n].double(), st["v"][s, :n].double()
            tk[s, n0:n0 + n] = _exact_turn(case, k, at, 1.0, "model", "pool", 1.0)
            tv[s, n0:n0 + n] = v
            if pages is not None:
                raw = _exact_turn(case, k, torch.zeros_like(at), 1.0, "model", "pool", 1.0)
                for b in range(n0 // B, (n0 + n + B - 1) // B):
                    lo, hi = max(b * B, n0), min(b * B + B, n0 + n)
                    for kv, x in ((0, raw), (1, v)):
                        pages[int(st["table"][s, b]), kv, :, :, lo - b * B:hi - b * B] = x[lo - n0:hi - n0].permute(1, 2, 0, 3)
        return (q, tk, tv) + ((pages,) if pages is not None else ())
    r, d = H // G, case["dim"]
    out, lse = st["out"].double(), st["lse"].double()
    for s in range(S):
        n, t, T = int(st["n_new"][s]), int(st["n_tail"][s]), int(st["n_sel"][s]) * B
        for layer in range(L):
            for g in range(G):
                K = torch.cat([st["k"][s, layer, g, :T], st["tail_k"][s, :t + n, layer, g]]).double()
                V = torch.cat([st["v"][s, layer, g, :T], st["tail_v"][s, :t + n, layer, g]]).double()
                for h in range(g * r, (g + 1) * r):
                    x = st["q"][s, :n, layer, h].double() @ K.T / math.sqrt(d)
                    x += torch.full((n, T + t + n), -math.inf, dtype=torch.float64, device="cuda").triu(T + t + 1)
                    z = torch.logsumexp(x, 1)
                    out[s, :n, layer, h] = (x - z.unsqueeze(1)).exp() @ V
                    lse[s, :n, layer, h] = z
    return out, lse
