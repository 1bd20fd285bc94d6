"""The calls on the cache's pages with stream= behind a busy current stream, from
two threads, and in CUDA graphs: tables, counts, lengths and cache bytes equal the
oracle's, as in tests/test_gpu_pages.py."""
import threading

import numpy as np
import pytest
import torch

from oracle import serving as S
from test_gpu_pages import Pool, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def busy(ms=20):
    """Work on the current stream that goes on using memory which has been given back already."""
    a = torch.ones((4096, 4096), device="cuda")
    for _ in range(ms):
        a = (a @ a).clamp_(-1, 1)
        for size in (512, 2048, 8192, 1 << 15, 1 << 17, 1 << 20):
            torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    return a


def grown(p, lens, n, parent):
    """What a reserve of n slots and a fork make of the oracle's side of a pool; the flags."""
    p.table, p.ref, f = S.reserve(p.table, p.ref, lens, n)
    new = np.asarray(lens) + np.asarray(n)
    p.table, p.ref, new, g = S.fork(p.table, p.ref, parent, new, [p.k, p.v])
    return new, f | g


@pytest.mark.parametrize("B,P", [(3, 5), (40, 30), (700, 12)])
def test_page_calls_beside_a_busy_stream(dreams, B, P):
    side = torch.cuda.Stream()
    for turn in range(4):
        p = Pool(dreams, B, P, B * P + B, layers=2, Hkv=2, D=64, seed=turn)
        rng = p.rng
        n = rng.integers(0, 64 * P - 64, B).astype(np.int32)
        parent = rng.integers(0, B, B).astype(np.int32)
        zero, gn, gp, new = i32(np.zeros(B)), i32(n), i32(parent), i32(np.zeros(B))
        torch.cuda.synchronize()
        keep = busy()
        dreams.kv_reserve(p.pool, zero, gn, status=p.st, stream=side)
        dreams.kv_fork(p.pool, gp, gn, new_kv_len=new, status=p.st, stream=side)
        side.synchronize()
        got, st = new.clone(), p.st.clone()
        del keep
        want, f = grown(p, np.zeros(B, np.int32), n, parent)
        np.testing.assert_array_equal(got.cpu().numpy(), want)
        assert int(st.item()) == f == 0
        p.same()


def test_results_beside_a_busy_stream(dreams):
    """The results that the calls make themselves."""
    g = torch.Generator().manual_seed(1)
    side = torch.cuda.Stream()
    p = Pool(dreams, 40, 6, 300, Hkv=2, D=64, seed=9)
    lens = p.rng.integers(80, 64 * 6 - 2, 40).astype(np.int32)
    p.reserve(np.zeros(40, np.int32), lens + 2)
    for x in (p.gk, p.gv):
        x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
    q = torch.randn((40, 2, 8, 64), generator=g).to(torch.bfloat16).cuda()
    gl, two, keep = i32(lens), i32(np.full(40, 2)), i32(np.tile(np.arange(5, 35), (40, 1)))
    ref, ref_lse = dreams.window_attention(q, p.kv, two, gl, 0.125, 100, 3, want_lse=True)
    for _ in range(4):
        torch.cuda.synchronize()
        held = busy(5)
        out, lse = dreams.window_attention(q, p.kv, two, gl, 0.125, 100, 3, want_lse=True, stream=side)
        new = dreams.kv_prune(dreams.KVCache(p.gk.clone(), p.gv.clone(), p.gt), keep, 5, 70, gl, stream=side)
        side.synchronize()
        assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
        assert torch.equal(new, gl - 40)
        del held


def test_argmax_beside_a_busy_stream(dreams):
    """Its workspace has to be zero-filled when it runs, on a stream that has made none yet too."""
    g = torch.Generator().manual_seed(2)
    for rows in (7, 80, 300):
        logits = torch.randn((rows, 50000), generator=g).cuda()
        arg = torch.argmax(logits, 1).to(torch.int32)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        held = busy(5)
        top = dreams.vocab_argmax(logits, stream=side)
        side.synchronize()
        assert torch.equal(top, arg)
        del held


def test_pools_of_two_threads(dreams):
    """Each thread has a pool and a stream of its own."""
    errors = []

    def work(seed):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                p = Pool(dreams, 20, 6, 200, Hkv=2, D=64, seed=seed)
                lens = np.zeros(20, np.int32)
                for turn in range(25):
                    n = np.minimum(64 * 6 - lens, p.rng.integers(0, 60, 20)).astype(np.int32)
                    assert p.reserve(lens, n) == 0
                    p.append(lens, n, 64)
                    lens, f = p.fork(p.rng.integers(0, 20, 20).astype(np.int32), lens + n)
                    assert f == 0
                    if turn % 6 == 5:
                        p.release(np.zeros(20), np.full(20, 64 * 6))
                        lens = np.zeros(20, np.int32)
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


@pytest.mark.parametrize("warm", [False, True])
def test_a_captured_step_hands_out_pages(dreams, warm):
    """Reserve, append, fork and release in a CUDA graph: each replay works on the tables as they are then, also when a
    larger pool has been used on the capture stream, and memory that was given back has been written to, in between."""
    B, P, T, H, D = 6, 9, 70, 2, 64
    p = Pool(dreams, B, P, 80, Hkv=H, D=D, seed=5)
    rng = p.rng
    lens = np.array([0, 10, 64, 100, 5, 30], np.int32)
    p.reserve(np.zeros(B, np.int32), lens)
    gl, gn, gp, new = i32(lens), i32(np.zeros(B)), i32(np.arange(B)), i32(np.zeros(B))
    top, rows = i32(np.full(B, 64 * P)), torch.zeros((B, T, 2, H, D), dtype=torch.bfloat16, device="cuda")

    def step():
        dreams.kv_reserve(p.pool, gl, gn, status=p.st)
        dreams.kv_append(p.kv, rows[:, :, 0], rows[:, :, 1], gl, gn, status=p.st)
        after = gl + gn
        dreams.kv_fork(p.pool, gp, after, new_kv_len=new, status=p.st)
        dreams.kv_release(p.pool, new, top, status=p.st)

    stream = torch.cuda.Stream()
    if warm:  # the same calls eagerly on that stream, nothing new and nothing moved
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        stream.synchronize()
        p.same()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for turn in range(5):
        n = rng.integers(0, T, B).astype(np.int32)
        if turn == 4:
            n[:] = 0
        parent = rng.integers(0, B, B).astype(np.int32)
        x = rng.integers(0, 1 << 15, (B, T, 2, H, D)).astype(np.int16)
        gl.copy_(i32(lens)), gn.copy_(i32(n)), gp.copy_(i32(parent))
        rows.copy_(torch.from_numpy(x).view(torch.bfloat16).cuda())
        with torch.cuda.stream(stream):  # a larger pool
            big = Pool(dreams, 50 + 20 * turn, 40, 60 * 40 * (turn + 1), seed=turn)
            m = np.full(50 + 20 * turn, 130, np.int32)
            big.reserve(m * 0, m)
            big.fork(np.zeros(len(m), np.int32), m)
            busy(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert int(p.st.item()) == 0
        # the oracle's side
        p.table, p.ref, f = S.reserve(p.table, p.ref, lens, n)
        assert f == 0
        for b in range(B):
            for t in range(n[b]):
                s = lens[b] + t
                p.k[0, p.table[b, s // 64], s % 64], p.v[0, p.table[b, s // 64], s % 64] = x[b, t, 0], x[b, t, 1]
        p.table, p.ref, lens, f = S.fork(p.table, p.ref, parent, lens + n, [p.k, p.v])
        assert f == 0
        p.table, p.ref, f = S.release(p.table, p.ref, lens, np.full(B, 64 * P))
        p.same(f)
        np.testing.assert_array_equal(new.cpu().numpy(), lens)
