"""Measured cases of the decode-side cache operators: what each computes, on which sizes, and what it must move.

  tree   attention of a tree of drafted tokens over the execution view (or straight over the selected pages) and the
         tail of tokens that do not fill a block yet (``Pool.view_tree_attend``, ``Pool.paged_tree_attend``)
  mass   decode attention over view and tail that also adds every view token's attention weight to an accumulator
         (``Pool.view_attend_mass``)
  evict  the tokens of each KV head with the largest accumulated weight, moved together into a smaller view
         (``Pool.view_evict``)

``run`` computes them in elementary torch operations in 32 bits; with ``own`` set it calls the package instead.
``exact`` computes them once more, in 64 bits, head by head.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128                      # head dimension of every configuration of this repository


# ------------------------------------------------------------------------------------------------ cases

def _tree(name, paged, sessions, layers, heads, kv_heads, block, blocks, drafted, tail, ragged):
    return {"name": name, "op": "tree", "paged": paged, "sessions": sessions, "layers": layers, "heads": heads,
            "kv_heads": kv_heads, "block": block, "blocks": blocks, "drafted": drafted, "tail": tail, "ragged": ragged}


def _mass(name, sessions, layers, heads, kv_heads, block, blocks, queries, tail, ragged):
    return {"name": name, "op": "mass", "sessions": sessions, "layers": layers, "heads": heads, "kv_heads": kv_heads,
            "block": block, "blocks": blocks, "drafted": queries, "tail": tail, "ragged": ragged}


def _evict(name, sessions, layers, heads, kv_heads, block, blocks, keep, sink, recent, ragged, zeros):
    return {"name": name, "op": "evict", "sessions": sessions, "layers": layers, "heads": heads, "kv_heads": kv_heads,
            "block": block, "blocks": blocks, "keep": keep, "sink": sink, "recent": recent, "ragged": ragged,
            "zeros": zeros}


def listed():
    return [
        # the 16,384-token history with its budget of 32 blocks: 8 drafted tokens, latency counts
        _tree("tree paged 2k, 8 drafted", True, 1, 1, 32, 8, 64, 32, 8, 37, False),
        # the 128K history with its budget of 512 blocks, read through the block table: a usual draft tree of 16
        _tree("tree paged 32k, 16 drafted", True, 1, 1, 32, 8, 64, 512, 16, 50, False),
        # the 1M history at the native window: 4,096 blocks in the view, the widest tree a mask row holds
        _tree("tree view 256k, 64 drafted", False, 1, 1, 32, 8, 64, 4096, 64, 63, False),
        # eight sessions of different lengths in one call, padded drafts, permuted pages
        _tree("tree paged batch 8, 12 drafted", True, 8, 1, 32, 8, 64, 1024, 12, 90, True),
        # a tail longer than many blocks, 32-token blocks, two layers, eight query heads on a KV head, odd tree
        _tree("tree view 24k, 33 drafted", False, 2, 2, 16, 2, 32, 777, 33, 1000, True),
        # one query token over a small view with its weights
        _mass("mass 2k, 1 query", 1, 1, 32, 8, 64, 32, 1, 20, False),
        # 1 + 3 drafted tokens over the native window
        _mass("mass 256k, 4 queries", 1, 1, 32, 8, 64, 4096, 4, 63, False),
        # eight sessions of different lengths, one query token each
        _mass("mass batch 8 64k, 1 query", 8, 1, 32, 8, 64, 1024, 1, 33, True),
        # a small view cut by a quarter
        _evict("evict 2k to 1.5k", 1, 1, 32, 8, 64, 32, 24, 4, 128, False, False),
        # the native window cut to half
        _evict("evict 256k to 128k", 1, 1, 32, 8, 64, 4096, 2048, 64, 1024, False, False),
        # eight sessions of different lengths; the shorter ones fit and stay whole
        _evict("evict batch 8 64k to 40k", 8, 1, 32, 8, 64, 1024, 640, 16, 300, True, False),
        # four layers, 32-token blocks, odd counts, most weights still zero: ties decide
        _evict("evict 23k to 7k, ties", 1, 4, 32, 4, 32, 723, 219, 5, 77, False, True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("tree", "mass", "evict"))
    sessions = _log(rng, 1, 8)
    layers = rng.choice((1, 1, 2, 3))
    kv_heads = rng.choice((1, 2, 4, 8))
    group = rng.choice((1, 2, 4, 4, 5, 8))
    block = rng.choice((16, 32, 64, 64, 128))
    # at most the native window of 262,144 tokens on 8 KV heads in all
    most = max(2, 262144 * 8 // (sessions * layers * kv_heads * block))
    blocks = _log(rng, 1, min(most, 8192 * 32 // block))
    ragged = sessions > 1 and rng.random() < 0.7
    if op == "tree":
        drafted = min(_log(rng, 1, 64), max(1, 256 // group))
        return _tree("", rng.random() < 0.5, sessions, layers, kv_heads * group, kv_heads, block, blocks, drafted,
                     rng.choice((0, _log(rng, 1, 300))), ragged)
    if op == "mass":
        return _mass("", sessions, layers, kv_heads * group, kv_heads, block, blocks, min(_log(rng, 1, 16), 64 // group),
                     rng.choice((0, _log(rng, 1, 300))), ragged)
    return _evict("", sessions, layers, kv_heads * group, kv_heads, block, blocks, max(1, int(blocks * rng.uniform(0.1, 1.1))),
                  rng.choice((0, _log(rng, 1, 64))), rng.choice((0, _log(rng, 1, 1024))), ragged, rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """Blocks in each session's view: equal, or from none to all of them in a fixed ragged pattern."""
    n, k = case["sessions"], case["blocks"]
    if not case["ragged"]:
        return [k] * n
    return [k if s == 0 else 0 if s == n - 1 and n > 2 else max(1, (k * (2 * s + 3)) // (2 * n + 3)) for s in range(n)]


def _queries_of(case):
    """Query tokens of each session: a padded batch where the case is ragged."""
    n, m = case["sessions"], case["drafted"]
    return [m if s == 0 or not case["ragged"] else max(1, m - (3 * s) % m) for s in range(n)]


def _tails_of(case):
    n, t = case["sessions"], case["tail"]
    return [t if s == 0 or not case["ragged"] else (t * (s + 1)) // (n + 1) for s in range(n)]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, u, n, blocks, block):
    """[sessions][heads][tokens][D] keys: N(0, 1), one block in sixteen shifted by three along its head's direction."""
    k = _normal(gen, n, u.shape[1], blocks * block, D)
    planted = torch.rand(n, 1, blocks, generator=gen, device="cuda") < 1.0 / 16
    k += 3.0 * planted.repeat_interleave(block, 2).unsqueeze(-1) * u.unsqueeze(2)
    return k.to(torch.bfloat16)


def _tree_masks(sessions, queries, most, rng_seed):
    """Ancestor bits (self included) of random trees: int64 [sessions][most]; rows behind a session's last are zero."""
    gen = torch.Generator().manual_seed(rng_seed)
    rows = []
    for s in range(sessions):
        bits = []
        for i in range(most):
            if i >= queries[s]:
                bits.append(0)
                continue
            parent = int(torch.randint(-1, max(1, i), (1,), generator=gen)) if i else -1
            bits.append((1 << i) | (bits[parent] if parent >= 0 else 0))
        rows.append([b - (1 << 64) if b >= (1 << 63) else b for b in bits])
    return torch.tensor(rows, dtype=torch.int64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    S, L, H, G, B, k = (case[x] for x in ("sessions", "layers", "heads", "kv_heads", "block", "blocks"))
    LG, dev = L * G, "cuda"
    n_sel = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)
    st = {"case": dict(case), "n_sel": n_sel}
    u = _normal(gen, S, LG, D)
    u /= u.norm(dim=-1, keepdim=True)
    if case["op"] == "evict":
        st["k"] = _keys(gen, u, S, k, B).view(S, L, G, k * B, D)
        st["v"] = _normal(gen, S, L, G, k * B, D).to(torch.bfloat16)
        # sums of attention weights: heavy-tailed, or mostly zero
        m = torch.exp(2.0 * _normal(gen, S, L, G, k * B)) / (k * B)
        if case["zeros"]:
            m *= torch.rand(S, L, G, k * B, generator=gen, device=dev) < 0.2
        st["mass"] = m
        keep = case["keep"]
        st["dst_k"] = torch.zeros(S, L, G, keep * B, D, dtype=torch.bfloat16, device=dev)
        st["dst_v"] = torch.zeros_like(st["dst_k"])
        st["dst_mass"] = torch.zeros(S, L, G, keep * B, device=dev)
        st["kept"] = torch.full((S, L, G, keep * B), -1, dtype=torch.int32, device=dev)
        st["n_out"] = torch.zeros(S, dtype=torch.int32, device=dev)
        pages = 1
    else:
        M, r = case["drafted"], H // G
        cap = case["tail"] + M
        q = _normal(gen, S, M, L, G, r, D) + math.sqrt(D) * u.view(S, 1, L, G, 1, D)
        st["q"] = q.view(S, M, L, H, D).to(torch.bfloat16)
        st["tail_k"] = _normal(gen, S, cap, L, G, D).to(torch.bfloat16)
        st["tail_v"] = _normal(gen, S, cap, L, G, D).to(torch.bfloat16)
        st["n_tail"] = torch.tensor(_tails_of(case), dtype=torch.int32, device=dev)
        st["n_q"] = torch.tensor(_queries_of(case), dtype=torch.int32, device=dev)
        st["out"] = torch.zeros(S, M, L, H, D, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.zeros(S, M, L, H, device=dev)
        pages = 1
        if case["op"] == "tree":
            st["mask"] = _tree_masks(S, _queries_of(case), M, int(seed)).to(dev)
        else:
            st["mass"] = torch.rand(S, L, G, k * B, generator=gen, device=dev) / (k * B)
        if case["op"] == "tree" and case["paged"]:
            # a history four times the budget; ascending ids, as the selector writes them
            hist = 4 * k
            st["hist_k"] = _keys(gen, u, S, hist, B).view(S, L, G, hist * B, D).permute(0, 3, 1, 2, 4).contiguous()
            st["hist_v"] = _normal(gen, S, hist * B, L, G, D).to(torch.bfloat16)
            st["sel"] = torch.rand(S, hist, generator=gen, device=dev).argsort(1)[:, :k].sort(1).values.to(torch.int32)
            pages = S * hist
        else:
            st["k"] = _keys(gen, u, S, k, B).view(S, L, G, k * B, D)
            st["v"] = _normal(gen, S, L, G, k * B, D).to(torch.bfloat16)
    if own:
        from paper_2609_04852_b200 import Pool, Tail, View
        st["pool"] = Pool(L, H, G, D, B, S, pages, max(1, pages // S), torch.cuda.current_device())
        if "hist_k" in st:
            perm = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed))).view(S, -1)
            for s in range(S):
                st["pool"].append_blocks(s, st["hist_k"][s], st["hist_v"][s], perm[s].tolist())
        if case["op"] == "evict":
            st["view"] = View(st["k"], st["v"], k * B)
            st["dst"] = View(st["dst_k"], st["dst_v"], case["keep"] * B)
        else:
            st["tail"] = Tail(st["tail_k"], st["tail_v"], st["n_tail"])
            if "k" in st:
                st["view"] = View(st["k"], st["v"], k * B)
    return st


# ------------------------------------------------------------------------------------------------ plain forms

def _heads_first(x):
    """[S][tokens][L][G][D] -> fp32 [S][L*G][tokens][D]"""
    return x.permute(0, 2, 3, 1, 4).flatten(1, 2).float()


def _attention(st, k, v, visible):
    """fp32 attention of q over [view | tail]: k, v [S][LG][T][D]; visible [S][M][tail tokens], or None: a chain.
    Returns the weights [S][LG][M*r][T + tail], outputs [S][LG][M*r][D] and log-sum-exp [S][LG][M*r]."""
    c = st["case"]
    S, L, H, G, M = c["sessions"], c["layers"], c["heads"], c["kv_heads"], c["drafted"]
    r, T = H // G, k.shape[2]
    q = st["q"].float().view(S, M, L, G, r, D).permute(0, 2, 3, 1, 4, 5).reshape(S, L * G, M * r, D)
    tk, tv = _heads_first(st["tail_k"]), _heads_first(st["tail_v"])
    cap = tk.shape[2]
    j = torch.arange(cap, device=q.device)
    drafted = j - st["n_tail"].view(S, 1)                                    # [S][cap]: index among the drafted tokens
    if visible is None:
        allowed = drafted.unsqueeze(1) <= torch.arange(M, device=q.device).view(1, M, 1)
    else:
        bit = (st["mask"].unsqueeze(2) >> drafted.clamp(0, 63).unsqueeze(1)) & 1
        allowed = (drafted.unsqueeze(1) < 0) | (bit != 0)
    allowed = allowed & (drafted < st["n_q"].view(S, 1)).unsqueeze(1)
    allowed = allowed.repeat_interleave(r, 1).unsqueeze(1)                    # [S][1][M*r][cap]
    live = (torch.arange(T, device=q.device) < (st["n_sel"] * c["block"]).view(S, 1)).view(S, 1, 1, T)
    scale = 1.0 / math.sqrt(D)
    x = torch.cat([(torch.matmul(q, k.transpose(2, 3)) * scale).masked_fill(~live, -math.inf),
                   (torch.matmul(q, tk.transpose(2, 3)) * scale).masked_fill(~allowed, -math.inf)], 3)
    top = x.amax(3, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = (x - top).exp_()
    del x
    z = p.sum(3, keepdim=True)
    p /= torch.where(z > 0, z, torch.ones_like(z))
    used = allowed.any(2).unsqueeze(3) if allowed.numel() else torch.zeros(S, 1, cap, 1, dtype=torch.bool, device=q.device)
    o = torch.matmul(p[..., :T], torch.where(live.view(S, 1, T, 1), v, torch.zeros((), device=v.device)))
    o += torch.matmul(p[..., T:], torch.where(used, tv, torch.zeros((), device=v.device)))
    return p, o, (top + z.log()).squeeze(3)


def _give(st, o, lse):
    """Rounded outputs in [S][M][L][H][D] order; rows of padded query tokens keep the zeros they had."""
    c = st["case"]
    S, L, H, G, M = c["sessions"], c["layers"], c["heads"], c["kv_heads"], c["drafted"]
    here = torch.arange(M, device=o.device).view(1, M, 1, 1) < st["n_q"].view(S, 1, 1, 1)
    o = o.view(S, L, G, M, H // G, D).permute(0, 3, 1, 2, 4, 5).reshape(S, M, L, H, D)
    lse = lse.view(S, L, G, M, H // G).permute(0, 3, 1, 2, 4).reshape(S, M, L, H)
    return (torch.where(here.unsqueeze(4), o, torch.zeros((), device=o.device)).to(torch.bfloat16),
            torch.where(here, lse, torch.zeros((), device=o.device)))


def _plain_tree(st):
    c = st["case"]
    if c["paged"]:
        S, L, G, B, k = c["sessions"], c["layers"], c["kv_heads"], c["block"], c["blocks"]
        at = st["sel"].long().view(S, k, 1, 1, 1, 1).expand(S, k, B, L, G, D)
        k_, v_ = (_heads_first(st[n].view(S, 4 * k, B, L, G, D).gather(1, at).view(S, k * B, L, G, D))
                  for n in ("hist_k", "hist_v"))
    else:
        k_, v_ = st["k"].flatten(1, 2).float(), st["v"].flatten(1, 2).float()
    _, o, lse = _attention(st, k_, v_, st["mask"])
    return _give(st, o, lse)


DECAY = 0.95                 # weight that the accumulator keeps from step to step


def _plain_mass(st):
    c = st["case"]
    S, L, H, G, M = c["sessions"], c["layers"], c["heads"], c["kv_heads"], c["drafted"]
    T = c["blocks"] * c["block"]
    p, o, lse = _attention(st, st["k"].flatten(1, 2).float(), st["v"].flatten(1, 2).float(), None)
    here = (torch.arange(M, device=o.device) < st["n_q"].view(S, 1)).repeat_interleave(H // G, 1).view(S, 1, -1, 1)
    w = (p[..., :T] * here).sum(2).view(S, L, G, T)
    live = (torch.arange(T, device=o.device) < (st["n_sel"] * c["block"]).view(S, 1)).view(S, 1, 1, T)
    st["mass"] = torch.where(live, st["mass"] * DECAY + w, st["mass"])
    return (*_give(st, o, lse), st["mass"])


def _plain_evict(st):
    c = st["case"]
    S, L, G, B, k, keep = (c[x] for x in ("sessions", "layers", "kv_heads", "block", "blocks", "keep"))
    T, C = k * B, keep * B
    t = torch.arange(T, device="cuda")
    n = (st["n_sel"].long() * B).view(S, 1, 1, 1)
    kept = n.clamp(max=C)
    sinks = kept.clamp(max=c["sink"])
    recents = (kept - sinks).clamp(max=c["recent"])
    # reserved tokens first, then the weights, then what lies behind the session's end
    rank = torch.where((t < sinks) | ((t >= n - recents) & (t < n)), math.inf, st["mass"])
    rank = torch.where(t < n, rank, -math.inf)
    order = rank.sort(dim=3, descending=True, stable=True).indices
    order = torch.where(t < kept, order, T)[..., :C].sort(3).values                      # ascending tokens, then T
    there = order < T
    at = order.clamp(max=T - 1)
    rows = at.unsqueeze(4).expand(*at.shape, D)
    zero = torch.zeros((), device="cuda")
    pad = (0, C - at.shape[3])
    dk, dv = (torch.nn.functional.pad(torch.where(there.unsqueeze(4), x.gather(3, rows), zero.to(x.dtype)), (0, 0) + pad)
              for x in (st["k"], st["v"]))
    dm = torch.nn.functional.pad(torch.where(there, st["mass"].gather(3, at), zero), pad)
    ids = torch.nn.functional.pad(torch.where(there, order, -1), pad, value=-1).to(torch.int32)
    return dk, dv, dm, ids, (kept // B).view(S).to(torch.int32)


# ------------------------------------------------------------------------------------------------ one pass

def run(st):
    c = st["case"]
    if not own:
        return {"tree": _plain_tree, "mass": _plain_mass, "evict": _plain_evict}[c["op"]](st)
    pool = st["pool"]
    if c["op"] == "tree" and c["paged"]:
        pool.paged_tree_attend(st["q"], st["sel"], st["n_sel"], st["tail"], st["out"], st["lse"], mask=st["mask"],
                               n_q=st["n_q"])
    elif c["op"] == "tree":
        pool.view_tree_attend(st["q"], st["view"], st["n_sel"], st["tail"], st["out"], st["lse"], mask=st["mask"],
                              n_q=st["n_q"])
    elif c["op"] == "mass":
        pool.view_attend_mass(st["q"], st["view"], st["n_sel"], st["mass"], st["out"], st["lse"], tail=st["tail"],
                              n_q=st["n_q"], decay=DECAY)
        return st["out"], st["lse"], st["mass"]
    else:
        pool.view_evict(st["view"], st["n_sel"], st["mass"], st["dst"], st["n_out"], st["dst_mass"], kept=st["kept"],
                        n_sink_tokens=c["sink"], n_recent_tokens=c["recent"])
        return st["dst_k"], st["dst_v"], st["dst_mass"], st["kept"], st["n_out"]
    return st["out"], st["lse"]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    S, L, H, G, B = (case[x] for x in ("sessions", "layers", "heads", "kv_heads", "block"))
    tokens = sum(_lengths(case)) * B
    LG = L * G
    if case["op"] == "evict":
        kept = sum(min(n, case["keep"]) for n in _lengths(case)) * B
        # weights read once; kept rows of K and V read and written, their weights and ids written
        return {"bytes": LG * (tokens * 4 + kept * (2 * 2 * D * 2 + 4 + 4)) + 8 * S, "flops": LG * tokens}
    queries, tails = _queries_of(case), _tails_of(case)
    seen = sum((n * B + t + m) for n, t, m in zip(_lengths(case), tails, queries))
    pairs = sum((n * B + t + m) * m for n, t, m in zip(_lengths(case), tails, queries))
    nbytes = LG * seen * 2 * D * 2 + sum(queries) * L * H * (D * 2 + D * 2 + 4) + 8 * sum(queries) + 12 * S
    if case["op"] == "mass":
        nbytes += LG * tokens * 8
    return {"bytes": nbytes, "flops": 4 * D * L * H * pairs}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_attention(st, s, lg):
    """One session and KV head in 64 bits: weights of view and tail tokens, outputs, log-sum-exp of its query rows."""
    c = st["case"]
    L, H, G, M, B = c["layers"], c["heads"], c["kv_heads"], c["drafted"], c["block"]
    layer, g, r = lg // G, lg % G, H // G
    n_tail, n_q, n_blk = int(st["n_tail"][s]), int(st["n_q"][s]), int(st["n_sel"][s])
    if "sel" in st:
        tok = (st["sel"][s, :n_blk].long().unsqueeze(1) * B + torch.arange(B, device="cuda")).reshape(-1)
        K, V = st["hist_k"][s, tok, layer, g].double(), st["hist_v"][s, tok, layer, g].double()
    else:
        K, V = st["k"][s, layer, g, :n_blk * B].double(), st["v"][s, layer, g, :n_blk * B].double()
    end = n_tail + n_q
    K = torch.cat([K, st["tail_k"][s, :end, layer, g].double()])
    V = torch.cat([V, st["tail_v"][s, :end, layer, g].double()])
    sees = torch.ones(n_q, K.shape[0], dtype=torch.bool)
    for i in range(n_q):
        bits = int(st["mask"][s, i]) if c["op"] == "tree" else (2 << i) - 1
        for jj in range(n_q):
            sees[i, n_blk * B + n_tail + jj] = bool((bits >> jj) & 1)
    sees = sees.to("cuda").repeat_interleave(r, 0)
    q = st["q"][s, :n_q, layer, g * r:(g + 1) * r].reshape(n_q * r, D).double()
    x = torch.where(sees, (q @ K.T) / math.sqrt(D), -math.inf)
    lse = torch.logsumexp(x, 1)
    w = torch.where(sees, (x - lse.unsqueeze(1)).exp(), 0.0)
    return w, w @ V, lse, n_blk * B


def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    S, L, H, G, B = (case[x] for x in ("sessions", "layers", "heads", "kv_heads", "block"))
    r = H // G
    if case["op"] == "evict":
        dk, dv = torch.zeros_like(st["dst_k"]).double(), torch.zeros_like(st["dst_v"]).double()
        dm = torch.zeros_like(st["dst_mass"]).double()
        for s in range(S):
            n = int(st["n_sel"][s]) * B
            keep = min(n, case["keep"] * B)
            sinks = min(case["sink"], keep)
            recents = min(case["recent"], keep - sinks)
            for lg in range(L * G):
                layer, g = lg // G, lg % G
                m = st["mass"][s, layer, g, :n].double()
                free = torch.ones(n, dtype=torch.bool, device="cuda")
                free[:sinks] = False
                free[n - recents:] = False
                left = keep - (n - int(free.sum()))
                ids = free.nonzero().squeeze(1)
                best = ids[torch.argsort(-m[ids], stable=True)[:left]]
                hold = ~free
                hold[best] = True
                ids = hold.nonzero().squeeze(1)
                dk[s, layer, g, :keep] = st["k"][s, layer, g, ids].double()
                dv[s, layer, g, :keep] = st["v"][s, layer, g, ids].double()
                dm[s, layer, g, :keep] = m[ids]
        return dk, dv, dm, None, None
    out, lse = torch.zeros_like(st["out"], dtype=torch.float64), torch.zeros_like(st["lse"], dtype=torch.float64)
    mass = st["mass"].double() if case["op"] == "mass" else None
    for s in range(S):
        n_q = int(st["n_q"][s])
        for lg in range(L * G):
            layer, g = lg // G, lg % G
            w, o, z, n = _exact_attention(st, s, lg)
            out[s, :n_q, layer, g * r:(g + 1) * r] = o.view(n_q, r, D)
            lse[s, :n_q, layer, g * r:(g + 1) * r] = z.view(n_q, r)
            if mass is not None:
                mass[s, layer, g, :n] = mass[s, layer, g, :n] * DECAY + w[:, :n].sum(0)
    return (out, lse) if mass is None else (out, lse, mass)
