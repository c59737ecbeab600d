"""The rotary table that a pool has after kvmem_set_rope: entry by entry, in fp32."""
import pytest
import torch

from paper_2609_04852_b200 import Pool, Rope

pytestmark = pytest.mark.gpu


def table(pool):
    """fp32 [positions][d / 2][cos | sin] as it lies at the end of the pool's storage."""
    n, half = pool.cfg.rope_max_positions, pool.cfg.head_dim // 2
    size = n * half * 8
    return pool.storage[pool.storage.numel() - (size + 255) // 256 * 256:][:size].view(torch.float32).view(n, half, 2)


@pytest.mark.parametrize("d,positions,theta", [(512, 92516, 5.0e5), (128, 4096, 1.0e4), (16, 9000, 1.0e6)])
def test_the_pools_own_form_again_is_the_table_it_was_created_with(d, positions, theta):
    """To the bit.  (The first: cos of pair 81 at position 92,515 lies within 2^-29 of the middle of two fp32 values.)"""
    pool = Pool(1, 1, 1, d, 64, 1, 1, 1, torch.cuda.current_device(), rope_max_positions=positions, rope_theta=theta)
    created = table(pool).clone()
    half = d // 2
    at = torch.tensor([0, 1, positions // 2, positions - 1])
    f = torch.tensor([theta ** (-2.0 * i / d) for i in range(half)], dtype=torch.float64)
    angle = at.double().view(-1, 1) * f
    want = torch.stack([angle.cos(), angle.sin()], -1)
    assert bool(((created[at.cuda()].cpu().double() - want).abs() <= 2.0 ** -24 * want.abs() * (1 + 2.0 ** -20) + 1e-12).all())
    for own in (Rope("interleaved"), None):                              # as it is
        pool.set_rope(own)
        assert torch.equal(table(pool).view(torch.int32), created.view(torch.int32))
    other = Rope("interleaved", 0, "linear", 2.0)
    for own in (None, Rope(), Rope("interleaved"), Rope("half", d)):
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            pool.set_rope(other)
            changed = table(pool).clone()
            pool.set_rope(own)
            again = table(pool).clone()
        st.synchronize()
        assert torch.equal(again.view(torch.int32), created.view(torch.int32)), own
        assert not torch.equal(changed, created)
        # half the angle: the row of an even position is that of half of it, as far as 64-bit angles and cosines agree in fp32
        n = positions // 2
        assert float((changed[0:2 * n:2] - created[:n]).abs().max()) <= 2.0 ** -23
    assert pool.device_status() == 0
