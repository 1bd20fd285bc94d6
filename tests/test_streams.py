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
    recorded = ()

    def record_stream(self, s):
        self.recorded += (s.cuda_stream,)


def gpu(t):
    return torch.Tensor._make_subclass(OnGpu, t)


class World:
    MAIN = 11  # the current stream's handle

    def __init__(self, patch):
        libbuild.build()
        dreams._lib()
        self.now, self.made, self.calls = self.MAIN, {}, []
        self.empties, self.fills = [], []  # the tensors made without a fill, and with one
        empty, zeros = torch.empty, torch.zeros

        def make(real):
            def f(*shape, device=None, **kw):
                t = gpu(real(*shape, **kw))
                self.made[t.data_ptr()] = self.now
                (self.empties if real is empty else self.fills).append((t, self.now))
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
        patch.setattr(dreams, "_WS_OUTGROWN", [], raising=False)

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


def _results(world):
    """Every call that makes its results, as functions of the stream."""
    z = lambda *s, dt=torch.bfloat16: gpu(torch.Tensor(*s).to(dt).zero_())  # noqa: E731
    f, i = (lambda *s: z(*s, dt=torch.float32)), (lambda *s: z(*s, dt=torch.int32))
    p, q, two, logits = world.pool(), z(2, 3, 4, 64), i(2), f(2, 3, 40)
    tree = dreams.Tree(i(2, 3), i(2, 3), two, two)
    p._by_stream.update({world.MAIN: i(1000), 22: i(1000)})
    return {
        "window_attention": lambda s: dreams.window_attention(q, p.kv, two, two, 0.1, 8, want_lse=True, stream=s),
        "kv_fork": lambda s: dreams.kv_fork(p, two, two, stream=s),
        "kv_prune": lambda s: dreams.kv_prune(p.kv, i(2, 3), 0, 4, two, stream=s),
        "tree_verify_attn": lambda s: dreams.tree_verify_attn(q, p.kv, tree, 0.1, want_lse=True, stream=s),
        "attention": lambda s: dreams.attention(q, p.kv, two, two, 0.1, dreams.ATTN_CAUSAL, want_lse=True, want_entropy=True, stream=s),
        "vocab_argmax": lambda s: dreams.vocab_argmax(f(3, 300000), stream=s),
        "vocab_sample": lambda s: dreams.vocab_sample(logits, 1.0, f(6), stream=s),
        "lm_head_argmax": lambda s: dreams.lm_head_argmax(z(3, 64), z(40, 64), want_max=True, stream=s),
        "visual_importance": lambda s: dreams.visual_importance(f(2, 2, 3, 9), 1, 5, 2, stream=s),
        "accept_path": lambda s: dreams.accept_path(i(2, 3), tree, 2, stream=s),
        "verify_step": lambda s: dreams.verify_step(logits, tree, p.kv, 2, stream=s),
        "verify_step_sampled": lambda s: dreams.verify_step_sampled(logits, tree, p.kv, 2, 1.0, f(2, 3), stream=s),
        "verify_step_speculative": lambda s: dreams.verify_step_speculative(logits, logits, tree, p.kv, 2, 1.0, f(2, 3), f(2, 3), stream=s)}


RESULTS = {"window_attention": 2, "kv_fork": 1, "kv_prune": 1, "tree_verify_attn": 2, "attention": 3, "vocab_argmax": 1, "vocab_sample": 1,
           "lm_head_argmax": 2, "visual_importance": 2, "accept_path": 4, "verify_step": 4, "verify_step_sampled": 4, "verify_step_speculative": 4}


@pytest.mark.parametrize("name", RESULTS)
def test_results_belong_to_the_stream_of_the_call(world, name):
    """Made under the call's stream, and held back for the current one, which reads them."""
    call = _results(world)[name]
    for s, handle in ((None, world.MAIN), (world.side(22), 22)):
        world.empties.clear()
        call(s)
        assert len(world.empties) == RESULTS[name]
        for t, under in world.empties:
            assert under == handle
            assert t.recorded == (() if s is None else (world.MAIN,))


@pytest.mark.parametrize("name", ["vocab_argmax", "vocab_sample", "lm_head_argmax", "visual_importance", "verify_step", "verify_step_sampled"])
def test_zero_filled_workspaces_are_filled_on_the_stream_of_the_call(world, name):
    call = _results(world)[name]
    for s, handle in ((None, world.MAIN), (world.side(22), 22)):
        world.fills.clear()
        call(s)
        assert [under for _, under in world.fills] == [handle]
        call(s)  # kept, and left zero-filled by the kernels
        assert len(world.fills) == 1


def test_an_outgrown_workspace_is_kept(world):
    """A captured call has its address. They do not pile up: each is at least twice as large as the one before."""
    sizes, kept = [], []
    for rows in (3, 5, 9, 40, 41, 42, 43, 200, 201):
        world.fills.clear()
        dreams.vocab_argmax(gpu(torch.Tensor(rows, 300000).zero_()))
        for t, _ in world.fills:
            sizes.append(t.numel())
            kept.append(t.data_ptr())
    alive = [t.data_ptr() for t in list(dreams._WS.values()) + dreams._WS_OUTGROWN]
    assert sorted(alive) == sorted(kept) and len(kept) > 1
    assert all(b >= 2 * a for a, b in zip(sizes, sizes[1:]))
