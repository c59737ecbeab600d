"""The calls that bring new tokens in, without a device: rotary frequencies against their formulas, sizes, and what is refused."""
import ctypes as C
import math

import pytest

from paper_2609_04852_b200 import KvmemError, PoolConfig, Rope, load_library
from paper_2609_04852_b200 import kvmem


def config(**kw):
    c = PoolConfig()
    base = dict(n_layers=1, n_q_heads=32, n_kv_heads=8, head_dim=128, block_tokens=64, max_sessions=4, max_blocks=8, max_blocks_per_session=8,
                device=0, rope_max_positions=4096, rope_theta=1.0e6)
    for k, v in {**base, **kw}.items():
        setattr(c, k, v)
    return c


def frequencies(cfg, rope):
    f = (C.c_double * (cfg.head_dim // 2))()
    rc = load_library().kvmem_rope_frequencies(C.byref(cfg), None if rope is None else C.byref(rope.struct()), f)
    if rc:
        raise KvmemError(rc, load_library().kvmem_last_error().decode())
    return list(f)


def test_plain_and_partial_frequencies():
    cfg = config()
    assert frequencies(cfg, None) == frequencies(cfg, Rope()) == frequencies(cfg, Rope("interleaved"))
    for i, f in enumerate(frequencies(cfg, None)):
        assert f == pytest.approx(1.0e6 ** (-i / 64), rel=1e-15)
    f = frequencies(cfg, Rope("half", 32))
    assert f[16:] == [0.0] * 48 and all(x == pytest.approx(1.0e6 ** (-2 * i / 32), rel=1e-15) for i, x in enumerate(f[:16]))


def test_scaled_frequencies():
    cfg = config()
    plain = frequencies(cfg, None)
    assert all(x == pytest.approx(y / 4, rel=1e-15) for x, y in zip(frequencies(cfg, Rope(scaling="linear", factor=4.0)), plain))
    base = frequencies(cfg, Rope(scaling="base", factor=4.0))
    assert base[0] == 1.0 and base[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)          # the slowest is divided by the factor, the fastest kept
    for scaling in ("ramp", "bands"):
        f = frequencies(cfg, Rope(scaling=scaling, factor=8.0, original_positions=4096.0))
        kept = [i for i in range(64) if f[i] == plain[i]]
        divided = [i for i in range(64) if f[i] == pytest.approx(plain[i] / 8, rel=1e-15)]
        assert kept == list(range(len(kept))) and divided == list(range(64 - len(divided), 64)) and 0 < len(kept) < 64 - len(divided) < 64
        assert all(a > b for a, b in zip(f, f[1:]))
        fast = 32.0 if scaling == "ramp" else 4.0
        turns = [4096.0 * p / (2 * math.pi) for p in plain]
        # (the ramp is laid through whole pairs, so its ends may lie a pair away)
        assert turns[len(kept)] < fast * (plain[0] / plain[1]) and turns[len(kept) - 1] > fast / (plain[0] / plain[1])
    # factor 1 changes nothing
    for scaling in ("linear", "base", "ramp", "bands"):
        assert all(x == pytest.approx(y, rel=1e-14) for x, y in zip(frequencies(cfg, Rope(scaling=scaling, factor=1.0, original_positions=4096.0)), plain))


def test_what_a_form_refuses():
    cfg = config()
    for rope, status in ((Rope("half", 24), kvmem.E_UNSUPPORTED), (Rope("half", 160), kvmem.E_INVALID), (Rope("half", -16), kvmem.E_INVALID),
                         (Rope(scaling="linear", factor=0.9), kvmem.E_INVALID), (Rope(scaling="base", factor=math.nan), kvmem.E_INVALID),
                         (Rope(scaling="ramp", factor=2.0), kvmem.E_INVALID), (Rope(scaling="bands", factor=2.0, original_positions=-5.0), kvmem.E_INVALID),
                         (Rope(scaling="ramp", factor=2.0, original_positions=64.0, turns_fast=1.0, turns_slow=1.0), kvmem.E_INVALID)):
        with pytest.raises(KvmemError) as e:
            frequencies(cfg, rope)
        assert e.value.status == status, rope
    with pytest.raises(KvmemError) as e:
        frequencies(config(rope_max_positions=0), Rope())
    assert e.value.status == kvmem.E_STATE
    lib = load_library()
    s = Rope().struct()
    for field, value in (("layout", 2), ("layout", -1), ("scaling", 5), ("scaling", -1)):
        bad = Rope().struct()
        setattr(bad, field, value)
        assert lib.kvmem_rope_frequencies(C.byref(cfg), C.byref(bad), (C.c_double * 64)()) == kvmem.E_INVALID
    assert lib.kvmem_rope_frequencies(C.byref(cfg), C.byref(s), None) == kvmem.E_INVALID
    assert lib.kvmem_rope_frequencies(C.byref(config(n_kv_heads=7)), C.byref(s), (C.c_double * 64)()) == kvmem.E_INVALID


def test_chunk_workspace_sizes():
    lib = load_library()

    def size(cfg, ns, M):
        return lib.kvmem_prefill_workspace_bytes(C.byref(cfg), ns, M)

    cfg = config()
    assert size(cfg, 1, 65) == size(cfg, 4, 100000) > 0                                     # the same whatever the call
    for M in (1, 17, 64):
        assert size(cfg, 3, M) == lib.kvmem_tree_workspace_bytes(C.byref(cfg), 3, M) > 0    # the decode kernel's
    many = config(n_q_heads=64)                                                             # 448 rows of a KV head and 2,560 in all
    assert size(many, 1, 56) == size(cfg, 1, 65) and size(many, 1, 55) == lib.kvmem_tree_workspace_bytes(C.byref(many), 1, 55)
    many = config(n_q_heads=64, n_kv_heads=1)
    assert size(many, 1, 40) == size(cfg, 1, 65) and size(many, 1, 39) == lib.kvmem_tree_workspace_bytes(C.byref(many), 1, 39)
    assert size(many, 2, 20) == size(cfg, 1, 65) and size(many, 5, 6) == lib.kvmem_tree_workspace_bytes(C.byref(many), 5, 6)
    many = config(n_q_heads=129, n_kv_heads=1)
    assert size(many, 1, 64) == lib.kvmem_tree_workspace_bytes(C.byref(many), 1, 64)
    for bad, ns, M in ((cfg, 0, 100), (cfg, 65536, 100), (cfg, 1, 0), (cfg, 1, -5), (config(head_dim=64), 1, 100), (config(n_q_heads=129, n_kv_heads=1), 1, 100),
                       (config(n_kv_heads=5), 1, 100), (cfg, 1, 65535 * 64 + 1), (cfg, 65535, 65535)):
        assert size(bad, ns, M) == 0 and lib.kvmem_last_error()
    assert size(config(n_q_heads=128, n_kv_heads=1), 1, 100) > 0
    assert size(cfg, 1, 65535 * 64) > 0


def test_calls_without_a_pool_fail_cleanly():
    lib = load_library()
    one = (C.c_int32 * 1)(1)
    assert lib.kvmem_set_rope(None, None, None) == kvmem.E_STATE
    assert lib.kvmem_rope_apply(None, None, 0, 0, 0, None, 0, 0, 0, 1, 1, None, 0, 1.0, None) == kvmem.E_STATE
    assert lib.kvmem_reserve_blocks(None, 0, 1, None, None) == kvmem.E_STATE
    assert lib.kvmem_rope_apply_call(None) == kvmem.E_INVALID and lib.kvmem_append_tokens_call(None) == kvmem.E_INVALID
    assert lib.kvmem_rope_apply_call(C.create_string_buffer(1024)) == kvmem.E_STATE                    # all zeros: no pool
    assert lib.kvmem_append_tokens_call(C.create_string_buffer(1024)) == kvmem.E_STATE
    assert lib.kvmem_session_reserved(None, 0) == kvmem.E_STATE
    assert lib.kvmem_append_tokens(None, 0, 1, 1, None, None, None, None, None, None, 0, 1.0, None, None, 0, None) == kvmem.E_STATE
    assert lib.kvmem_commit_blocks(None, 0, 1, one, None, None) == kvmem.E_STATE
    assert lib.kvmem_view_prefill_attend(None, 1, None, 100, None, None, None, 64, None, None, 0.0, None, None, None, 0, None) == kvmem.E_STATE
    assert lib.kvmem_get_pages(None, C.byref(C.c_void_p())) == kvmem.E_STATE


def test_names_of_forms():
    for bad in (Rope("thirds"), Rope("half", 0, "magic")):
        with pytest.raises(ValueError):
            bad.struct()
