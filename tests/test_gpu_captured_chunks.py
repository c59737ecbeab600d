"""A serving loop's step captured as it is written: new tokens appended, attended, made committed ones, all in one graph that is replayed
chunk after chunk.  Lengths are read on the device and sums are joined in one order, so the replays give the bits of the plain calls."""
import pytest
import torch

from paper_2609_04852_b200 import Rope, Tail
from test_gpu_tokens import ints, make_pool, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 12, 150])
def test_append_attend_and_count_in_one_graph(M):
    L, H, G, B, D, ns, steps = 1, 8, 2, 32, 128, 2, 4
    x = randn(5, steps, ns, M, L, H + 2 * G, D)
    results = []
    for captured in (False, True):
        pool = make_pool(L, H, G, D, B, ns, 30, 2048, Rope("interleaved", 64))
        for s in range(ns):
            pool.reserve_blocks(s, 30)
        view = pool.new_view(ns, 3 * B)
        view.k.copy_(randn(6, *view.k.shape)); view.v.copy_(randn(7, *view.v.shape))
        n_sel, n_new = ints([3, 2]), ints([M, M // 2 + 1])
        tail = Tail(*(torch.zeros(ns, steps * M + 9, L, G, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)), ints([4, 9]))
        new = torch.zeros_like(x[0])
        q, k, v = new[..., :H, :], new[..., H:H + G, :], new[..., H + G:, :]
        q_rot, out = (torch.zeros(ns, M, L, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lse = torch.zeros(ns, M, L, H, device="cuda")

        def step():
            pool.append_tokens(k, v, tail, q=q, q_out=q_rot, n_new=n_new, n_sel=n_sel, pages=True)
            pool.view_prefill_attend(q_rot, view, n_sel, tail, out, lse, n_q=n_new)
            tail.n_tokens.add_(n_new)

        run = step
        if captured:
            step()                                          # the workspace is there from here on
            tail.n_tokens.copy_(ints([4, 9]))
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            run = g.replay
        got = []
        for i in range(steps):
            new.copy_(x[i])
            run()
            n = [M, M // 2 + 1]
            got += [t[s, :n[s]].clone() for t in (q_rot, out, lse) for s in range(ns)]
        ends = tail.n_tokens.tolist()
        assert ends == [4 + steps * M, 9 + steps * (M // 2 + 1)] and pool.device_status() == 0
        got += [t[s, lo:e].clone() for t in (tail.k, tail.v) for s, (lo, e) in enumerate(zip((4, 9), ends))]
        assert all(bool(t.isfinite().all()) for t in got)
        results.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*results))
