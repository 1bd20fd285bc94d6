"""Pools of 8-bit pages at the boundary (no GPU): a fork of full pages takes no cache, and
no call on bf16 rows takes an 8-bit one."""
import ctypes

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from test_kv8_streams import world  # noqa: F401
from test_streams import gpu
from test_serving_abi import INV, P, WS, cache, lib, needs_no_gpu, pool  # noqa: F401


def codes(D):
    return gpu(torch.Tensor(4, 64, 2, D).to(torch.uint8).zero_().view(torch.float8_e4m3fn))


@needs_no_gpu
def test_a_fork_without_a_cache_is_checked_like_any_other(lib):  # noqa: F811
    r = ctypes.byref(pool())
    need = lib.dreams_kv_fork_workspace_size(r)
    for ws, n in ((None, need), (P, need - 1), (P + 4, need)):
        assert lib.dreams_kv_fork(None, r, P, P, P, ws, n, None, None) == WS
    for a in ((None, P, P), (P, None, P), (P, P, None), (P + 1, P, P), (P, P + 2, P), (P, P, P + 3)):
        assert lib.dreams_kv_fork(None, r, *a, P, need, None, None) == INV
    for p in (pool(page_table=None), pool(B=0), pool(num_pages=0)):
        assert lib.dreams_kv_fork(None, ctypes.byref(p), P, P, P, P, 1 << 30, None, None) == INV
    assert lib.dreams_kv_fork(ctypes.byref(cache(k=None)), r, P, P, P, P, need, None, None) == INV


def test_a_fork_of_8_bit_pages_hands_over_no_cache(world):  # noqa: F811
    p8 = dreams.PagePool(world.kv8, world.z(4, dt=torch.int32))
    p16 = dreams.PagePool(world.kv, world.z(4, dt=torch.int32))
    for pool8, p in ((True, p8), (False, p16)):
        dreams.kv_fork(p, world.ints(2), world.ints(2))
        name, _, args = world.calls[-1]
        assert name == "dreams_kv_fork" and (args[0] is None) == pool8


@pytest.mark.parametrize("D", [64, 128])
def test_calls_on_16_bit_rows_refuse_an_8_bit_cache(world, D):  # noqa: F811
    """Taken for one of bf16 rows, its codes would be read in pairs and overwritten."""
    z, i = world.z, world.ints
    c = lambda: codes(D)  # noqa: E731
    kv8 = dreams.KV8Cache(c(), c(), z(4, 2, 2, dt=torch.int16), z(2, 2, dt=torch.int32))
    kv = dreams.KVCache(z(4, 64, 2, D), z(4, 64, 2, D), z(2, 2, dt=torch.int32))
    q, n, r = z(2, 3, 4, D), z(2, 3, 2, D), dreams.Rotary(z(32, dt=torch.int64))
    tree = dreams.Tree(z(2, 3, dt=torch.int32), z(2, 3, dt=torch.int32), i(2), i(2))
    logits = z(2, 3, 8)
    u = lambda: z(2, 3, dt=torch.float32)  # noqa: E731
    calls = {
        "window_attention": lambda kv: dreams.window_attention(q, kv, i(2), i(2), 0.1, 8),
        "kv_append": lambda kv: dreams.kv_append(kv, n, n, i(2), i(2)),
        "kv_append_rope": lambda kv: dreams.kv_append_rope(kv, n, n, r, i(2), i(2), q=q),
        "kv_prune": lambda kv: dreams.kv_prune(kv, z(2, 1, dt=torch.int32), 0, 2, i(2)),
        "kv_quantize": lambda kv: dreams.kv_quantize(kv, kv8, i(2), i(2)),
        "kv8_attention": lambda kv: dreams.kv8_attention(q, kv8, kv, i(2), i(2), i(2), 0.1),
        "tree_verify_attn": lambda kv: dreams.tree_verify_attn(q, kv, tree, 0.1, workspace=z(1 << 20, dt=torch.uint8)),
        "kv_compact": lambda kv: dreams.kv_compact(kv, i(2), i(2), z(2, 3, dt=torch.int32)),
        "verify_step": lambda kv: dreams.verify_step(logits, tree, kv, 3, workspace=z(1 << 20, dt=torch.uint8)),
        "verify_step_speculative": lambda kv: dreams.verify_step_speculative(logits, logits, tree, kv, 3, 1.0, u(), u()),
    }
    for name, f in calls.items():
        f(kv)
        world.calls.clear()
        with pytest.raises(TypeError):
            f(kv8)
        assert not world.calls, name
    for f in (lambda: dreams.kv_quantize(kv, kv, i(2), i(2)), lambda: dreams.kv8_attention(q, kv, kv, i(2), i(2), i(2), 0.1)):
        with pytest.raises(TypeError):
            f()
    assert not world.calls
