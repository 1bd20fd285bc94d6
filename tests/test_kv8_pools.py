"""Pools of 8-bit pages at the boundary (no GPU): a fork of full pages takes no cache."""
import ctypes

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from test_kv8_streams import world  # noqa: F401
from test_serving_abi import INV, P, WS, cache, lib, needs_no_gpu, pool  # noqa: F401


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
