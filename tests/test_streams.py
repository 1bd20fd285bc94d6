"""Whose memory the binding works in, without a GPU: tensors that say they are on
one, a caching allocator that notes the stream each tensor is made under, and
launches that are noted instead of made."""
import contextlib
import types

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from paper_2606_00535_gb300 import build as libbuild

CUDA = torch.device("cuda", 0)


class OnGpu(torch.Tensor):
    """A CPU tensor that says it is on the GPU."""
    device = CUDA


def gpu(t):
    return torch.Tensor._make_subclass(OnGpu, t)


class World:
    MAIN = 11  # the current stream's handle

    def __init__(self, patch):
        libbuild.build()
        dreams._lib()
        self.now, self.made, self.calls = self.MAIN, {}, []
        empty, zeros = torch.empty, torch.zeros

        def make(real):
            def f(*shape, device=None, **kw):
                t = gpu(real(*shape, **kw))
                self.made[t.data_ptr()] = self.now
                return t
            return f

        @contextlib.contextmanager
        def stream(s):
            before, self.now = self.now, self.now if s is None else s.cuda_stream
            yield
            self.now = before

        patch.setattr(torch, "empty", make(empty))
        patch.setattr(torch, "zeros", make(zeros))
        patch.setattr(torch.cuda, "stream", stream)
        patch.setattr(torch.cuda, "current_stream", lambda dev=None: types.SimpleNamespace(cuda_stream=self.now, device=CUDA))
        patch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.now, raising=False)
        patch.setattr(dreams, "_launch", lambda name, dev, stream, *a: self.calls.append((name, stream, a)))
        patch.setattr(dreams, "_call", lambda name, dev, *a: self.calls.append((name, None, a)))
        patch.setattr(dreams, "_WS", {})

    def side(self, handle):
        return types.SimpleNamespace(cuda_stream=handle, device=CUDA)

    def pool(self, pages=4, B=2, P=2):
        z = lambda *s, dt=torch.bfloat16: gpu(torch.Tensor(*s).to(dt).zero_())  # noqa: E731
        kv = dreams.KVCache(z(pages, 64, 2, 64), z(pages, 64, 2, 64), z(B, P, dt=torch.int32))
        return dreams.PagePool(kv, z(pages, dt=torch.int32))

    def ints(self, n):
        return gpu(torch.Tensor(n).to(torch.int32).zero_())

    def workspace(self):
        """(address, bytes) that the last page call was given."""
        name, _, a = self.calls[-1]
        return tuple(a[3:5]) if name == "dreams_kv_reserve" else tuple(a[5:7])


@pytest.fixture
def world(monkeypatch):
    return World(monkeypatch)


CALLS = {"reserve": lambda p, i, **kw: dreams.kv_reserve(p, i, i, **kw), "fork": lambda p, i, **kw: dreams.kv_fork(p, i, i, new_kv_len=i, **kw)}


@pytest.mark.parametrize("call", CALLS)
def test_a_pools_workspace_belongs_to_the_stream_it_is_used_on(world, call):
    p, i = world.pool(), world.ints(2)
    for s, handle in ((None, world.MAIN), (world.side(22), 22), (world.side(33), 33), (world.side(22), 22)):
        CALLS[call](p, i, stream=s)
        at, n = world.workspace()
        assert world.made[at] == handle
        assert n >= max(p._reserve_bytes, p._fork_bytes)


@pytest.mark.parametrize("call", CALLS)
def test_a_pools_workspace_stays_while_the_pool_lives(world, call):
    """A captured call has its address: neither another pool's call nor a larger one's takes it away or shares it."""
    p, i = world.pool(), world.ints(2)
    CALLS[call](p, i)
    at, n = world.workspace()
    other, large = world.pool(), world.pool(pages=500, B=60, P=40)
    for q, j in ((other, i), (large, world.ints(60)), (p, i)):
        CALLS[call](q, j)
        a, m = world.workspace()
        assert (q is p) == (a == at)
        assert a == at or a + m <= at or at + n <= a  # (the first is still alive: its address is not given out again)


@pytest.mark.parametrize("call", CALLS)
def test_a_callers_workspace_is_used(world, call):
    p, i = world.pool(), world.ints(2)
    mine = gpu(torch.Tensor(1 << 12).to(torch.int32))
    CALLS[call](p, i, workspace=mine, stream=world.side(22))
    at, n = world.workspace()
    assert (at if isinstance(at, int) else at.value) == mine.data_ptr() and n == mine.numel() * 4
