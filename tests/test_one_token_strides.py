"""Strides of dimensions of size one, which no address uses: neither the library nor
the binding refuses a call for them (no GPU)."""
import ctypes

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from test_serving_abi import INV, P, cache, lib, needs_no_gpu  # noqa: F401
from test_streams import gpu, world  # noqa: F401


@needs_no_gpu
@pytest.mark.parametrize("st", [64, 0, -8, 3])
def test_the_library_ignores_the_token_stride_of_one_token(lib, st):  # noqa: F811
    """Past the checks the launch fails, as there is no GPU: any answer but the refusal of an argument."""
    kv = cache(D=64)
    for B, sb in ((3, 4 * 64), (1, 0)):
        assert lib.dreams_window_attention(P, sb, st, ctypes.byref(kv), 0, None, P, P, B, 1, 4, 0.1, 4, 0, P, None, None, None) != INV
        assert lib.dreams_kv_append(ctypes.byref(kv), 0, P, P, sb, st, P, P, B, 1, None, None) != INV
    # two tokens use it, and several sequences use theirs
    assert lib.dreams_window_attention(P, 8 * 64, st, ctypes.byref(kv), 0, None, P, P, 3, 2, 4, 0.1, 4, 0, P, None, None, None) == INV
    assert lib.dreams_kv_append(ctypes.byref(kv), 0, P, P, 8 * 64, st, P, P, 3, 2, None, None) == INV
    assert lib.dreams_window_attention(P, 64, st, ctypes.byref(kv), 0, None, P, P, 3, 1, 4, 0.1, 4, 0, P, None, None, None) == INV
    assert lib.dreams_kv_append(ctypes.byref(kv), 0, P, P, 64, st, P, P, 3, 1, None, None) == INV


def test_the_binding_takes_heads_first_layouts(world):  # noqa: F811
    z = lambda *s, dt=torch.bfloat16: gpu(torch.zeros(s, dtype=dt))  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    kv = dreams.KVCache(z(2, 64, 2, 64), z(2, 64, 2, 64))
    mqa = dreams.KVCache(z(2, 64, 1, 64), z(2, 64, 1, 64))
    # one token, stored [B, H, 1, D]
    dreams.window_attention(z(2, 4, 1, 64).transpose(1, 2), kv, i(2), i(2), 0.1, 8)
    assert world.calls[-1][2][1:3] == (4 * 64, 4 * 64)
    dreams.kv_append(kv, z(2, 2, 1, 64).transpose(1, 2), z(2, 2, 1, 64).transpose(1, 2), i(2), i(2))
    assert world.calls[-1][2][4:6] == (2 * 64, 2 * 64)
    # one KV head, stored [B, 1, T, D], beside a dense one; one sequence with an odd stride
    dreams.kv_append(mqa, z(2, 1, 5, 64).transpose(1, 2), z(2, 5, 1, 64), i(2), i(2))
    assert world.calls[-1][2][4:6] == (5 * 64, 64)
    dreams.kv_append(kv, z(3, 5, 2, 64)[:1], z(5, 3, 2, 64).transpose(0, 1)[:1].contiguous(), i(2), i(2))
    dreams.kv_append(kv, z(1, 3, 2, 64), torch.as_strided(z(3 * 128), (1, 3, 2, 64), (8, 128, 64, 1)), i(2), i(2))
    n = len(world.calls)
    for k, v in ((z(2, 2, 3, 64).transpose(1, 2),) * 2, (z(2, 3, 2, 64), z(2, 2, 3, 64).transpose(1, 2)), (z(2, 3, 2, 64), z(2, 6, 2, 64)[:, ::2])):
        with pytest.raises(ValueError):
            dreams.kv_append(kv, k, v, i(2), i(2))
    with pytest.raises(ValueError):
        dreams.window_attention(z(2, 4, 2, 64).transpose(1, 2), kv, i(2), i(2), 0.1, 8)
    assert len(world.calls) == n
