"""kv_fork on pools of 8-bit pages: tables, counts and lengths equal the oracle's, the codes
and their powers are not touched, and a length that is no multiple of 64 changes nothing."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from test_gpu_kv8 import codes8
from test_gpu_pages import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


class Pool8:
    def __init__(self, dreams, B, P, pages, lens, layers=2):
        """Sequences of these lengths on pages of their own."""
        self.d, self.B = dreams, B
        self.k, self.v = codes8((layers, pages, 64, 2, 64)), codes8((layers, pages, 64, 2, 64))
        self.exps = torch.randint(-20, 20, (layers, pages, 2, 2), dtype=torch.int16, device="cuda")
        self.gt = torch.empty((B, P), dtype=torch.int32, device="cuda")
        self.pool = dreams.PagePool.empty(dreams.KV8Cache(self.k, self.v, self.exps, self.gt))
        self.st = i32([0])
        dreams.kv_reserve(self.pool, i32([0] * B), i32(lens), status=self.st)
        self.table, self.ref = self.gt.cpu().numpy(), self.pool.refcount.cpu().numpy()
        assert int(self.st) == 0
        self.before = [x.view(torch.uint8).clone() for x in (self.k, self.v, self.exps)]

    def fork(self, parent, lens, alias=False):
        g = i32(lens)
        new = self.d.kv_fork(self.pool, i32(parent), g, new_kv_len=g if alias else None, status=self.st)
        if any(q >= 0 and lens[q] % 64 != 0 for q in parent):
            want, flags = np.asarray(lens), S.BAD_KV_LEN
        else:
            self.table, self.ref, want, flags = S.fork(self.table, self.ref, parent, lens, [])
        torch.cuda.synchronize()
        assert int(self.st) == flags and new.tolist() == want.tolist()
        self.st.zero_()
        np.testing.assert_array_equal(self.gt.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.pool.refcount.cpu().numpy(), self.ref)
        for x, y in zip((self.k, self.v, self.exps), self.before):
            assert torch.equal(x.view(torch.uint8), y)
        return want.tolist(), flags


def test_full_pages_are_shared(dreams):
    p = Pool8(dreams, 4, 5, 20, [320, 64, 0, 128])
    lens, _ = p.fork([0, 0, 1, -1], [320, 64, 0, 128])
    assert lens == [320, 320, 64, 0]
    lens, _ = p.fork([2, 1, 1, 1], [256, 320, 64, 0], alias=True)
    assert lens == [64, 320, 320, 320]


@pytest.mark.parametrize("bad", [100, 1, 63, 65, 319])
def test_other_lengths_change_nothing(dreams, bad):
    p = Pool8(dreams, 3, 5, 20, [320, 128, 64])
    for parent in ([0, 0, 1], [0, 1, 2], [2, 1, 0]):
        assert p.fork(parent, [bad, 128, 64])[1] == dreams.DATA_BAD_KV_LEN
    assert p.fork([1, 1, 2], [bad, 128, 64])[1] == 0  # nobody's parent: not looked at


@pytest.mark.parametrize("B,P", [(20, 34), (300, 40), (1200, 9)])
def test_tables_of_every_size(dreams, B, P):
    rng = np.random.default_rng(B)
    lens = [64 * int(n) for n in rng.integers(0, P + 1, B)]
    p = Pool8(dreams, B, P, sum(lens) // 64 + 1, lens, layers=1)
    lens, flags = p.fork([int(x) for x in rng.integers(-1, B, B)], lens)
    assert flags == 0
    odd = list(lens)
    odd[B // 2] = 30
    assert p.fork(list(range(B)), odd)[1] == dreams.DATA_BAD_KV_LEN


def test_replayed_from_a_graph(dreams):
    p = Pool8(dreams, 3, 5, 20, [320, 128, 64])
    parent, lens, new = i32([0, 0, 1]), i32([320, 128, 64]), i32([0, 0, 0])
    ws = torch.empty(p.pool._fork_bytes, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dreams.kv_fork(p.pool, parent, lens, new_kv_len=new, workspace=ws, status=p.st)
    lens.copy_(i32([256, 130, 64]))
    graph.replay()
    assert new.tolist() == [256, 130, 64] and int(p.st) == dreams.DATA_BAD_KV_LEN
    np.testing.assert_array_equal(p.gt.cpu().numpy(), p.table)
    lens.copy_(i32([256, 128, 64]))
    p.st.zero_()
    graph.replay()
    table, ref, want, _ = S.fork(p.table, p.ref, [0, 0, 1], [256, 128, 64], [])
    assert new.tolist() == want.tolist() and int(p.st) == 0
    np.testing.assert_array_equal(p.gt.cpu().numpy(), table)
    np.testing.assert_array_equal(p.pool.refcount.cpu().numpy(), ref)
