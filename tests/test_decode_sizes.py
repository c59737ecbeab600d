"""The decode calls' sizes and refusals that need no device: workspaces, limits, calls without a pool."""
import ctypes as C

import pytest

from paper_2609_04852_b200 import PoolConfig, Tail, load_library
from paper_2609_04852_b200 import kvmem

CFG = PoolConfig(2, 32, 8, 128, 64, 8, 1, 1, 0)


def test_workspaces_grow_with_what_they_hold():
    lib = load_library()
    tree = lambda ns, m: lib.kvmem_tree_workspace_bytes(C.byref(CFG), ns, m)             # noqa: E731
    mass = lambda ns, m, cap: lib.kvmem_mass_workspace_bytes(C.byref(CFG), ns, m, cap)   # noqa: E731
    heads, segments = 16, 148 + 16
    # partial sums of both slots: fp32 rows of 128 per segment, at most 128 rows a slot
    assert tree(1, 1) >= segments * 2 * 4 * 128 * 4
    assert tree(1, 1) < tree(1, 16) < tree(2, 16) < tree(2, 64)
    # the logits of the weights: 4 bytes per row, head and token of capacity
    assert mass(1, 4, 4096) - tree(1, 4) >= heads * 16 * 4096 * 4
    assert mass(1, 4, 8192) - mass(1, 4, 4096) == heads * 16 * 4096 * 4
    ev = lib.kvmem_evict_workspace_bytes(C.byref(CFG), 3, 10)
    assert ev >= 3 * 16 * 10 * 64 * 4 + 3 * 8


@pytest.mark.parametrize("args", [(0, 1), (1, 0), (1, 65), (-1, 4), (65536, 1)])
def test_sizes_refuse_what_the_calls_refuse(args):
    lib = load_library()
    assert lib.kvmem_tree_workspace_bytes(C.byref(CFG), *args) == 0 and lib.kvmem_last_error()
    assert lib.kvmem_mass_workspace_bytes(C.byref(CFG), *args, 64) == 0


def test_sizes_refuse_bad_configurations_and_lengths():
    lib = load_library()
    bad = PoolConfig(2, 32, 5, 128, 64, 8, 1, 1, 0)
    assert lib.kvmem_tree_workspace_bytes(C.byref(bad), 1, 1) == 0 and lib.kvmem_tree_workspace_bytes(None, 1, 1) == 0
    assert lib.kvmem_mass_workspace_bytes(C.byref(CFG), 1, 1, 0) == 0
    assert lib.kvmem_evict_workspace_bytes(C.byref(CFG), 1, 0) == 0 and lib.kvmem_evict_workspace_bytes(C.byref(CFG), 0, 1) == 0
    assert lib.kvmem_evict_workspace_bytes(None, 1, 1) == 0


def test_calls_without_a_pool_fail_cleanly():
    lib = load_library()
    assert lib.kvmem_view_tree_attend(None, 1, None, 1, None, None, None, None, 64, None, None, 0.0, None, None, None, 0, None) == kvmem.E_STATE
    assert lib.kvmem_paged_tree_attend(None, 0, 1, None, 1, None, None, None, 1, None, None, 0.0, None, None, None, 0, None) == kvmem.E_STATE
    assert lib.kvmem_view_attend_mass(None, 1, None, 1, None, None, None, 64, None, None, 0.0, None, 1.0, None, None, None, 0, None) == kvmem.E_STATE
    assert lib.kvmem_view_evict(None, 1, None, None, 64, None, None, 1, 0, 0, None, None, 64, None, None, None, None, 0, None) == kvmem.E_STATE
    assert b"pool" in lib.kvmem_last_error()


def test_the_tail_struct_is_the_headers():
    # pointer, pointer, int32 (padded), pointer
    assert C.sizeof(kvmem.TailStruct) == 32 and kvmem.TailStruct.n_tokens.offset == 24 and kvmem.TailStruct.cap_tokens.offset == 16
    assert [f.name for f in __import__("dataclasses").fields(Tail)] == ["k", "v", "n_tokens"]
