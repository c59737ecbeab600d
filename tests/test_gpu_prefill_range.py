"""Values near the end of fp32's range in a chunk's attention over long views: sums of weighted values stay finite as long as the
view is, whatever the logits do after a row's first tokens.  Bounds: those of the chunk attention's tests."""
import pytest
import torch

from test_gpu_prefill import D, Chunk

pytestmark = pytest.mark.gpu


def level(c, steps):
    """Queries of one dim, the view's first 64 keys at a logit of 0 and the others at those of `steps` in turn, in units of the scale."""
    c.q.zero_(); c.q[..., 0] = 1.0
    T = c.k.shape[3]
    at = torch.tensor(steps, device="cuda")[torch.arange(T, device="cuda") * len(steps) // T]
    at[:64] = 0.0
    c.k.zero_(); c.k[..., 0] = at.to(torch.bfloat16)
    c.tk.zero_()
    v = 2.0 ** 111 * (1.0 + torch.arange(D, device="cuda") / 128.0) * (1.0 - 2.0 * (torch.arange(D, device="cuda") % 2))
    c.v[:] = v.to(torch.bfloat16); c.tv[:] = v.to(torch.bfloat16)


# one item over all SMs (many short shares to join); items with long shares, whole and cut
SIZES = [dict(M=100, H=1, G=1, lens=(1024,), tails=(5,)), dict(M=1280, H=32, G=8, lens=(1024,), tails=(5,)), dict(M=70, H=4, G=1, lens=(2048,), tails=None)]


@pytest.mark.parametrize("i", range(len(SIZES)))
@pytest.mark.parametrize("steps", [(1.0,), (1.0, 1.25, 1.5, 1.75), (0.0,), (1.0, 0.0, -1.0, 1.0)])
def test_weighted_values_stay_finite_over_long_views(i, steps):
    """A weight of 2^5.98 for all tokens but the first 64: half a tile of them sums to just under 2^12, all of them to 2^22."""
    c = Chunk(seed=i, scale=5.98 / 1.4426950408889634, extra=0, **SIZES[i])
    level(c, steps)
    c.call()
    assert bool(c.out.isfinite().all()) and bool(c.lse.isfinite().all())
    c.check()
