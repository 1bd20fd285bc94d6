"""kv8_attention for several sequences whose rows are pairs of blocks of 128: on clusters
of two CTAs that cut the longest pairs between them (up to a pair for seven SMs in
eight), and on CTAs that walk over pairs ordered by their tiles (above that). Against
the fp64 oracle, with the bounds that test_gpu_kv8.py derives."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from test_gpu_kv8 import Case, U, i32

pytestmark = pytest.mark.gpu
ALL = 2 ** 31 - 1


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    yield d
    d.test_set_stall(0, -1)


def full(lens, back=0):
    return [max(0, L // 64 - back) * 64 for L in lens]


# With 8 KV heads and 4 query heads each, a pair is 64 tokens: 48 pairs, each cut in half if it is long enough
CUT = [0, 63, 700, 1500, 1021, 1300]
# 96 pairs: 56 clusters have one pair, 20 a long and a short one
BESIDE = [1500, 90, 1400, 0, 1100, 700, 1200, 300, 1450, 500, 63, 900]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [CUT, BESIDE, [800] * 6, [640] * 12], ids=["cut", "beside", "equal", "equal beside"])
@pytest.mark.parametrize("tree", [True, False])
def test_lengths(dreams, D, lens, tree):
    n = ([64, 33, 1, 60, 0, 47] * 2)[:len(lens)]
    c = Case(len(lens) + D, 32, 8, D, lens, n, full(lens, 1), tree=tree, T_max=64)
    c.check(c.run(dreams), n=6)


@pytest.mark.parametrize("G,Hkv,T", [(1, 8, 256), (2, 16, 100), (7, 4, 100), (16, 4, 16), (128, 4, 2)])
def test_head_layouts(dreams, G, Hkv, T):
    lens = [900, 200, 1300, 640, 30, 1100] if T <= 100 else [900, 200, 1300]
    n = [T, T - 1, (T + 1) // 2, T, 1, T][:len(lens)]
    c = Case(G, G * Hkv, Hkv, 128, lens, n, full(lens), T_max=T)
    c.check(c.run(dreams), n=6)


@pytest.mark.parametrize("window,sinks", [(1, 0), (70, 4), (500, 100), (700, 0), (701, 65), (1000, 640), (ALL, ALL)])
@pytest.mark.parametrize("kind", ["tree", "chunk"])
def test_windows_and_sinks(dreams, window, sinks, kind):
    """The two blocks of a pair begin at different tiles, with a gap behind the sinks that only one of them reads."""
    lens = [1500, 640, 0, 1333, 1000, 777]
    T = 64 if kind == "tree" else 130
    n = [T, T, T, 40, 33, T]
    c = Case(window % 1000 + sinks % 100, 32, 8, 64, lens, n, full(lens, 2), window, sinks, tree=kind == "tree", T_max=T)
    c.check(c.run(dreams), n=8)


@pytest.mark.parametrize("D", [64, 128])
def test_many_pairs(dreams, D):
    """More pairs than clusters: CTAs walk over them, forth and back."""
    lens = [100, 1300, 600, 0]
    c = Case(D, 32, 8, D, lens, [400, 230, 333, 399], full(lens, 1), T_max=400)
    c.check(c.run(dreams), n=20)


def test_many_sequences(dreams):
    """More pairs than are put in order."""
    lens = [int(x) for x in np.random.default_rng(3).integers(0, 200, 300)]
    c = Case(3, 8, 1, 64, lens, [33 - b % 20 for b in range(300)], full(lens), T_max=33)
    c.check(c.run(dreams), n=2)


@pytest.mark.parametrize("lens", [CUT, BESIDE], ids=["cut", "beside"])
def test_what_only_some_rows_see(dreams, lens):
    """An infinity or a NaN in a node's V, in the part of either CTA: rows off its path keep their values."""
    for bad in (float("inf"), float("nan")):
        c = Case(5, 32, 8, 128, lens, [64] * len(lens), full(lens), tree=True)
        for b, L in enumerate(lens):
            c.parent[b] = [-1] + [0] * 63
            page, row = divmod(L + 7, 64)
            c.v[0, int(c.table[b, page]), row] = bad
        out, lse = c.run(dreams)
        assert not torch.isfinite(out[:, 7].float()).any()
        rng = np.random.default_rng(0)
        for b, L in enumerate(lens):
            K, V = c.vals[0, 0, b], c.vals[1, 0, b]
            sel = [(int(t), int(h)) for t, h in zip(rng.choice([t for t in range(64) if t != 7], 4, replace=False), rng.integers(0, 32, 4))]
            ref = S.window_rows(c.q[b].double().numpy(), lambda s, g: (K[s, g], V[s, g]), L, c.scale, ALL, 0, lambda h: h // 4, c.parent[b], sel)
            for (t, h), (o, a, z) in zip(sel, ref):
                assert (np.abs(out[b, t, h].double().cpu().numpy() - o) <= 1.02 * U * (np.abs(o) + a) + 2e-4 * a + 1e-6).all()


@pytest.mark.parametrize("up", [4, 6])
@pytest.mark.parametrize("big", [0, 80])
def test_scores_that_outgrow_the_first(dreams, up, big):
    """K of the later pages 2^up times as large: sums beyond what a part's reference allows, with values of V up to 2^big,
    in one part or in both."""
    lens = [1500, 1100, 640, 900, 1280, 1400]
    c = Case(up, 32, 8, 64, lens, [64, 20, 33, 64, 64, 50], full(lens), tree=True)
    for b, L in enumerate(lens):
        for e in range(L // 128, L // 64):
            z = int(c.table8[b, e])
            c.exps[0, z, :, 0] += up
            c.vals[0, 0, b, 64 * e:64 * e + 64] *= 2.0 ** up
            c.exps[0, z, :, 1] += big
            c.vals[1, 0, b, 64 * e:64 * e + 64] *= 2.0 ** big
    out, lse = (x.double().cpu().numpy() for x in c.run(dreams))
    rng = np.random.default_rng(1)
    for b, L in enumerate(lens):
        K, V, q = c.vals[0, 0, b], c.vals[1, 0, b], c.q[b].double().numpy()
        sel = [(int(t), int(h)) for t, h in zip(rng.integers(0, c.q_len[b], 6), rng.integers(0, 32, 6))]
        ref = S.window_rows(q, lambda s, g: (K[s, g], V[s, g]), L, c.scale, ALL, 0, lambda h: h // 4, c.parent[b], sel)
        for (t, h), (o, a, z) in zip(sel, ref):
            # D products summed in f32: off by at most D 2^-24 of their magnitudes' sum, so weights by twice that share
            e = 2 * 64 * 2.0 ** -24 * c.scale * (np.abs(K[:L + 64, h // 4]) @ np.abs(q[t, h])).max()
            assert (np.abs(out[b, t, h] - o) <= 1.02 * U * (np.abs(o) + a) + (2e-4 + 2 * e) * a + 1e-6).all(), (b, t, h)
            assert abs(lse[b, t, h] - z) <= 1e-4 + 1e-6 * abs(z) + e


@pytest.mark.parametrize("lens", [CUT, BESIDE], ids=["cut", "beside"])
def test_bad_data(dreams, lens):
    """Bad sequences, long or short, are flagged and left untouched, the others computed."""
    T = 64
    for s in (1, 3):
        for field, bad, want in (("len8", 32, dreams.DATA_BAD_KV_LEN), ("len8", 10 ** 6 * 64, dreams.DATA_BAD_KV_LEN), ("kv_len", -1, dreams.DATA_BAD_KV_LEN),
                                 ("kv_len", 10 ** 6, dreams.DATA_BAD_KV_LEN), ("q_len", -1, dreams.DATA_BAD_TREE_LEN), ("q_len", T + 1, dreams.DATA_BAD_TREE_LEN),
                                 ("parent", 5, dreams.DATA_BAD_PARENT)):
            c = Case(s, 32, 8, 64, list(lens), [T] * len(lens), full(lens), tree=True)
            if field == "parent":
                c.parent[s][5] = bad
            else:
                getattr(c, field)[s] = bad
            got = c.run(dreams, want)
            c.q_len[s] = 0
            c.check(got, n=1, skip=(s,))


@pytest.mark.parametrize("lens", [CUT, BESIDE], ids=["cut", "beside"])
def test_missing_and_marked_pages(dreams, lens):
    for s, e in ((3, 2), (3, 0), (5, 10)) if lens is CUT else ((0, 1), (0, 20), (7, 3)):
        c = Case(7, 32, 8, 128, lens, [64] * len(lens), full(lens), tree=True)
        c.table8[s, e] = -1
        got = c.run(dreams, dreams.DATA_BAD_PAGE)
        c.vals[:, 0, s, 64 * e:64 * e + 64] = 0.0  # reads as zeros
        c.check(got, n=4)
        for j in (0, 1):
            c = Case(7, 32, 8, 128, lens, [64] * len(lens), full(lens), tree=True, mark={(s, e, j)})
            c.check(c.run(dreams), n=4, nan=lambda b, t: b == s)


def test_graphs_with_other_lengths(dreams):
    """A captured call plans anew at each replay; the same call twice gives the same bits."""
    cases = [Case(s, 32, 8, 128, lens, [64] * 12, full(lens), tree=True) for s, lens in ((1, BESIDE), (2, BESIDE[::-1]))]
    want = [c.run(dreams) for c in cases]

    def inputs(c):
        return [c.q, c.k, c.v, c.table, c.k8, c.v8, c.exps, c.table8, *(torch.tensor(x, dtype=torch.int32) for x in (c.q_len, c.kv_len, c.len8, c.parent))]

    held = [x.cuda() for x in inputs(cases[0])]
    q, k, v, table, k8, v8, exps, table8, ql, kl, l8, par = held
    kv, kv8 = dreams.KVCache(k, v, table), dreams.KV8Cache(k8.view(torch.float8_e4m3fn), v8.view(torch.float8_e4m3fn), exps, table8)
    dreams.kv8_attention(q, kv8, kv, ql, kl, l8, cases[0].scale, parent=par)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = dreams.kv8_attention(q, kv8, kv, ql, kl, l8, cases[0].scale, parent=par, want_lse=True)
    for i in (1, 0, 0, 1):
        for x, y in zip(held, inputs(cases[i])):
            assert x.shape == y.shape
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("stall_at", [0, 1, 4])
def test_waits_of_one_or_both_parts_run_out(dreams, D, stall_at):
    """9 tiles a pair, 5 of them one CTA's and 4 the other's: from the fifth on, one of them alone gives up, and neither
    writes a row. The next call is bit-identical to the one before."""
    lens = [9 * 128 - 64] * 6
    c = Case(D, 32, 8, D, lens, [64] * 6, full(lens), tree=True)
    want = c.run(dreams)
    try:
        dreams.test_set_stall(dreams.TEST_ATTENTION, stall_at, 20_000_000)
        out, lse = c.run(dreams, dreams.DATA_TIMEOUT)
    finally:
        dreams.test_set_stall(0, -1)
    assert (out == 7.0).all() and (lse == 7.0).all()
    got = c.run(dreams)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.check(got, n=2)
