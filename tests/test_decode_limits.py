"""Limits of the decode calls: what a call refuses for its size has no workspace size either, and a call that is too large
says KVMEM_E_UNSUPPORTED, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2609_04852_b200 import Pool, PoolConfig, load_library
from paper_2609_04852_b200 import kvmem


def config(H=32, G=8, L=2, d=128, B=64):
    return PoolConfig(L, H, G, d, B, 8, 1, 1, 0)


def sizes():
    lib = load_library()
    return (lambda cfg, ns, m: lib.kvmem_tree_workspace_bytes(C.byref(cfg), ns, m),
            lambda cfg, ns, m, cap: lib.kvmem_mass_workspace_bytes(C.byref(cfg), ns, m, cap),
            lambda cfg, ns, keep: lib.kvmem_evict_workspace_bytes(C.byref(cfg), ns, keep))


def test_rows_per_kv_head():
    tree, mass, _ = sizes()
    wide = config(H=1024, G=1)
    assert tree(wide, 1, 64) > 0                                         # 65,536 rows
    assert tree(config(H=1025, G=1), 1, 64) == 0 and b"65536" in load_library().kvmem_last_error()
    assert tree(config(H=1 << 30, G=1), 1, 64) == 0                      # 2^36 rows
    assert mass(config(H=64, G=1), 1, 1, 64) > 0 and mass(config(H=4, G=1), 1, 16, 64) > 0
    assert mass(config(H=65, G=1), 1, 1, 64) == 0 and b"64 rows" in load_library().kvmem_last_error()
    assert mass(config(H=5, G=1), 1, 13, 64) == 0


def test_capacities_of_the_weights_view():
    _, mass, _ = sizes()
    assert mass(config(), 1, 1, 1 << 23) > 0 and mass(config(), 1, 1, (1 << 23) + 64) == 0
    assert mass(config(B=48), 1, 1, 96) > 0
    for cap in (32, 65, 96, -64):                                        # not whole blocks of 64 tokens
        assert mass(config(), 1, 1, cap) == 0


def test_head_dimension():
    tree, mass, evict = sizes()
    for d in (64, 256):
        assert tree(config(d=d), 1, 1) == 0 and mass(config(d=d), 1, 1, 64) == 0 and evict(config(d=d), 1, 1) == 0
        assert b"head_dim 128" in load_library().kvmem_last_error()


def test_the_line_of_tiles():
    """2^30 units: a unit per 128 tokens of capacity and three per KV head; 16 heads a session, 65,536 tiles of 128 tokens."""
    tree, mass, _ = sizes()
    assert 1023 * 16 * (65536 + 3) < 1 << 30 <= 1024 * 16 * (65536 + 3)
    assert mass(config(), 1023, 1, 1 << 23) > 0
    assert mass(config(), 1024, 1, 1 << 23) == 0 and b"2^30" in load_library().kvmem_last_error()
    # heads alone: a tile and three units each (a tile of two and eight above 128 rows), row groups of 256
    assert tree(config(L=256, G=16, H=16), 65535, 1) > 0 and tree(config(L=256, G=17, H=17), 65535, 1) == 0      # 2^28 and 2^28 * 17 / 16
    assert tree(config(L=256, G=6, H=24), 65535, 64) > 0 and tree(config(L=256, G=7, H=28), 65535, 64) == 0
    assert tree(config(L=256, G=3, H=24), 65535, 64) > 0 and tree(config(L=256, G=4, H=32), 65535, 64) == 0      # two row groups
    assert tree(config(L=256, G=1 << 30, H=1 << 30), 65535, 1) == 0


def test_kept_tokens():
    _, _, evict = sizes()
    assert evict(config(), 1, (1 << 25) - 1) > 0 and evict(config(), 1, 1 << 25) == 0              # 2^31 tokens
    assert evict(config(L=256, G=15, H=15), 65535, 1) > 0 and evict(config(L=256, G=17, H=17), 65535, 1) == 0   # 2^28 heads


@pytest.mark.gpu
def test_calls_beyond_the_limits_are_refused_as_unsupported():
    """Sizes that only a host check looks at: the capacities claim far more than any buffer here has."""
    pool = Pool(1, 8, 2, 128, 64, 1, 4, 4, 0)
    lib, ns = pool.lib, 65535
    dev = torch.device("cuda", 0)
    big = torch.zeros(4 << 20, dtype=torch.uint8, device=dev)
    zeros = torch.zeros(ns, dtype=torch.int32, device=dev)
    p, z, cap = big.data_ptr(), zeros.data_ptr(), 1 << 24
    tail = kvmem.TailStruct(p, p, 1 << 14, z)
    stream = torch.cuda.current_stream().cuda_stream
    for M in (1, 64):
        assert lib.kvmem_view_tree_attend(pool.handle, ns, p, M, z, None, p, p, cap, z, None, 0.0, p, p, p, 1 << 62, stream) == kvmem.E_UNSUPPORTED
        assert b"2^30" in lib.kvmem_last_error()
        assert lib.kvmem_paged_tree_attend(pool.handle, 0, 1, p, M, z, None, z, 1, z, None, 0.0, p, p, p, 0, stream) == kvmem.E_CAPACITY
    assert lib.kvmem_view_tree_attend(pool.handle, ns, p, 1, z, None, p, p, 1 << 20, z, None, 0.0, p, p, p, 1 << 62, stream) == kvmem.E_UNSUPPORTED
    assert lib.kvmem_view_tree_attend(pool.handle, ns, p, 1, z, None, p, p, (1 << 20) - (1 << 14), z, tail, 0.0, p, p, p, 1 << 62, stream) == kvmem.E_UNSUPPORTED
    assert lib.kvmem_view_attend_mass(pool.handle, ns, p, 1, z, p, p, 1 << 23, z, None, 0.0, p, 1.0, p, p, p, 1 << 62, stream) == kvmem.E_UNSUPPORTED
    assert lib.kvmem_view_evict(pool.handle, ns, p, p, cap, z, p, cap // 64, 0, 0, p, p, cap, p, None, z, p, 1 << 62, stream) == kvmem.E_UNSUPPORTED
    torch.cuda.synchronize()
    assert bool((big == 0).all()) and bool((zeros == 0).all())


@pytest.mark.gpu
def test_python_calls_report_the_calls_own_status():
    """A size that has no workspace still reaches the call, which names the reason."""
    dev = torch.device("cuda", 0)
    for H, G, d, M, status in ((130, 2, 128, 1, kvmem.E_UNSUPPORTED), (8, 2, 64, 1, kvmem.E_UNSUPPORTED), (8, 2, 128, 65, kvmem.E_INVALID)):
        pool = Pool(1, H, G, d, 64, 1, 1, 1, 0)
        q = torch.zeros(1, M, 1, H, d, dtype=torch.bfloat16, device=dev)
        view = kvmem.View(*(torch.zeros(1, 1, G, 64, d, dtype=torch.bfloat16, device=dev) for _ in range(2)), 64)
        n, mass, lse = torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros(1, 1, G, 64, device=dev), torch.zeros(1, M, 1, H, device=dev)
        with pytest.raises(kvmem.KvmemError) as e:
            pool.view_attend_mass(q, view, n, mass, torch.zeros_like(q), lse)
        assert e.value.status == status
        with pytest.raises(kvmem.KvmemError) as e:
            pool.view_evict(view, n, mass, kvmem.View(torch.zeros_like(view.k), torch.zeros_like(view.k), 64), n.clone(), torch.zeros_like(mass),
                            keep_blocks=0 if d == 128 else 1)
        assert e.value.status == (kvmem.E_INVALID if d == 128 else kvmem.E_UNSUPPORTED)


@pytest.mark.gpu
def test_session_ranges_whose_end_passes_32_bits_are_refused():
    pool = Pool(1, 8, 2, 128, 64, 4, 4, 4, 0)
    lib, last = pool.lib, (1 << 31) - 1
    dev = torch.device("cuda", 0)
    big, n = torch.zeros(1 << 20, dtype=torch.uint8, device=dev), torch.zeros(4, dtype=torch.int32, device=dev)
    p, z, stream = big.data_ptr(), n.data_ptr(), torch.cuda.current_stream().cuda_stream
    for first, ns in ((last, 1), (last, 4), (1, last), (last, last), (4, 1), (1, 4), (-1, 1), (0, 0), (0, -1)):
        assert lib.kvmem_paged_tree_attend(pool.handle, first, ns, p, 1, z, None, z, 1, z, None, 0.0, p, p, p, 1 << 20, stream) == kvmem.E_INVALID, (first, ns)
    assert lib.kvmem_session_blocks(pool.handle, last) == kvmem.E_INVALID and lib.kvmem_session_reset(pool.handle, last, stream) == kvmem.E_INVALID
    assert lib.kvmem_session_blocks(pool.handle, 3) == 0
    torch.cuda.synchronize()
    assert bool((big == 0).all())
