"""Whose memory rope, kv_append_rope, kv_quantize and kv8_attention work in: results that
a call makes are made on the stream it runs on, arguments are handed over as they are
(no GPU: the launches are recorded, the tensors only say that they are on one)."""
import pytest
import torch

import paper_2606_00535_gb300 as dreams
from test_streams import World, gpu


@pytest.fixture
def world(monkeypatch):
    w = World(monkeypatch)
    z = lambda *s, dt=torch.bfloat16: gpu(torch.Tensor(*s).to(dt).zero_())  # noqa: E731
    w.z = z
    w.kv = dreams.KVCache(z(4, 64, 2, 64), z(4, 64, 2, 64), z(2, 2, dt=torch.int32))
    c = lambda: gpu(torch.Tensor(4, 64, 2, 64).to(torch.uint8).zero_().view(torch.float8_e4m3fn))  # noqa: E731
    w.kv8 = dreams.KV8Cache(c(), c(), z(4, 2, 2, dt=torch.int16), z(2, 2, dt=torch.int32))
    w.rotary = dreams.Rotary(z(32, dt=torch.int64))
    return w


CALLS = {
    "dreams_rope": lambda w, **kw: dreams.rope(w.z(2, 3, 4, 64), w.rotary, **kw),
    "dreams_kv_append_rope": lambda w, **kw: dreams.kv_append_rope(w.kv, w.z(2, 3, 2, 64), w.z(2, 3, 2, 64), w.rotary, w.ints(2), w.ints(2),
                                                                   q=w.z(2, 3, 4, 64), **kw),
    "dreams_kv_quantize": lambda w, **kw: dreams.kv_quantize(w.kv, w.kv8, w.ints(2), w.ints(2), **kw),
    "dreams_kv8_attention": lambda w, **kw: dreams.kv8_attention(w.z(2, 3, 4, 64), w.kv8, w.kv, w.ints(2), w.ints(2), w.ints(2), 0.1, want_lse=True, **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_results_belong_to_the_stream_of_the_call(world, name):
    for stream in (None, world.side(77)):
        r = CALLS[name](world, stream=stream)
        called, given, _ = world.calls[-1]
        assert called == name and given is stream
        for t in r if isinstance(r, tuple) else (r,):
            assert world.made[t.data_ptr()] == (World.MAIN if stream is None else 77)


@pytest.mark.parametrize("name,kw", [("dreams_rope", "out"), ("dreams_kv_append_rope", "q_out"), ("dreams_kv8_attention", "out")])
def test_a_given_result_is_written_and_returned(world, name, kw):
    out = world.z(2, 3, 4, 64)
    r = CALLS[name](world, **{kw: out})
    assert (r[0] if isinstance(r, tuple) else r) is out and out.data_ptr() in world.calls[-1][2]


def test_rope_in_place_hands_over_one_pointer(world):
    x = world.z(2, 3, 4, 64)
    assert dreams.rope(x, world.rotary, out=x) is x
    assert world.calls[-1][2].count(x.data_ptr()) == 2


def test_an_8_bit_cache_is_a_pool_of_pages_like_any_other(world):
    """reserve, release and fork work on its pages as bytes: rows of the codes' size."""
    pool = dreams.PagePool(world.kv8, world.z(4, dt=torch.int32))
    dreams.kv_reserve(pool, world.ints(2), world.ints(2))
    name, _, args = world.calls[-1]
    assert name == "dreams_kv_reserve"
    with pytest.raises(ValueError):
        dreams.PagePool(world.kv8, world.z(3, dt=torch.int32))
