"""GPU parity of sliding-window attention with sinks (dreams_window_attention)
against the fp64 oracle, on bf16-rounded inputs.

Tolerance. Probabilities enter the PV product as bf16 and the output is rounded
to bf16 once: each costs at most u = 2^-8 relative (8 significant bits), so with A = sum_j a_j |V_j|
an element may be off by u (|O| + A). Scores and sums are f32: D products of
unit-normal values and the exponential cost at most about 1e-4 of A together.
The bound is 1.02 u (|O| + A) + 2e-4 A + 1e-6. The log-sum-exp carries the
scores' f32 error alone: 1e-4 + 1e-6 |lse|."""
import numpy as np
import pytest
import torch

from oracle import serving as S

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def _tree(rng, T, T_max):
    par = [-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, T)]
    return (par + [-1] * T_max)[:T_max]


class Case:
    """One seeded problem on the CPU: a cache (contiguous, or pages in random
    order with everything behind the window of the first query left out), queries,
    and the rows it is checked at."""

    def __init__(self, seed, Hq, Hkv, D, kv_len, q_len, window, sinks, tree=False, paged=False, T_max=None, layers=1, layer=0,
                 kscale=1.0):
        rng = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.D = len(kv_len), Hq, Hkv, D
        self.kv_len, self.q_len, self.window, self.sinks = kv_len, q_len, window, sinks
        self.T_max = T_max or max(1, max(q_len))
        self.cap = -(-max(L + n for L, n in zip(kv_len, q_len)) // 64) * 64 + 64
        self.layers, self.layer, self.scale = layers, layer, D ** -0.5
        self.parent = [_tree(rng, max(1, n), self.T_max) for n in q_len] if tree else None
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn((self.B, self.T_max, Hq, D), generator=g).to(torch.bfloat16)
        shape = (layers, self.B, self.cap, Hkv, D)
        self.k = (torch.randn(shape, generator=g) * kscale).to(torch.bfloat16)
        self.v = torch.randn(shape, generator=g).to(torch.bfloat16)
        self.table = None
        if paged:
            P = self.cap // 64
            self.table = torch.full((self.B, P), -1, dtype=torch.int32)
            use = [(b, e) for b in range(self.B) for e in range(P)
                   if e * 64 < kv_len[b] + q_len[b] and (64 * e + 64 > kv_len[b] - window + 1 or 64 * e < sinks)]
            ids = rng.permutation(len(use) + 3)
            self.kp = torch.full((layers, len(use) + 3, 64, Hkv, D), float("nan"), dtype=torch.bfloat16)
            self.vp = self.kp.clone()
            for i, (b, e) in enumerate(use):
                self.table[b, e] = int(ids[i])
                self.kp[:, ids[i]] = self.k[:, b, 64 * e:64 * e + 64]
                self.vp[:, ids[i]] = self.v[:, b, 64 * e:64 * e + 64]

    def run(self, dreams, want=0, q=None, **kw):
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        k, v = (self.k, self.v) if self.table is None else (self.kp, self.vp)
        kv = dreams.KVCache(k.cuda(), v.cuda(), None if self.table is None else self.table.cuda())
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full((self.B, self.T_max, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.B, self.T_max, self.Hq), 7.0, dtype=torch.float32, device="cuda")
        dreams.window_attention(self.q.cuda() if q is None else q, kv, i32(self.q_len), i32(self.kv_len), self.scale, self.window,
                                self.sinks, parent=None if self.parent is None else i32(self.parent), layer=self.layer, out=out,
                                lse=lse, status=st, **kw)
        torch.cuda.synchronize()
        assert int(st.item()) == want
        return out, lse

    def check(self, got, n=60, seed=0, skip=()):
        out, lse = got[0].float().cpu().numpy().astype(np.float64), got[1].cpu().numpy().astype(np.float64)
        rng = np.random.default_rng(seed)
        G = self.Hq // self.Hkv
        for b in range(self.B):
            assert (out[b, self.q_len[b]:] == 7.0).all() and (lse[b, self.q_len[b]:] == 7.0).all()
            sel = [(t, h) for t in range(self.q_len[b]) for h in range(self.Hq) if (b, t) not in skip]
            if len(sel) > n:  # the ends and some between
                sel = [sel[0], sel[-1]] + [sel[i] for i in rng.choice(len(sel), n, replace=False)]
            K, V = (x[self.layer, b].double().numpy() for x in (self.k, self.v))
            par = None if self.parent is None else self.parent[b]
            ref = S.window_rows(self.q[b].double().numpy(), lambda s, g: (K[s, g], V[s, g]), self.kv_len[b], self.scale, self.window,
                                self.sinks, lambda h: h // G, par, sel)
            for (t, h), (o, a, z) in zip(sel, ref):
                err = np.abs(out[b, t, h] - o)
                tol = 1.02 * U * (np.abs(o) + a) + 2e-4 * a + 1e-6
                assert (err <= tol).all(), (b, t, h, float((err / tol).max()))
                assert abs(lse[b, t, h] - z) <= 1e-4 + 1e-6 * abs(z), (b, t, h, lse[b, t, h], z)


HEADS = [(28, 4, 128), (32, 8, 128), (8, 8, 128), (4, 4, 64), (16, 1, 64), (10, 2, 128), (128, 1, 128)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("paged", [False, True])
def test_single_tokens(dreams, Hq, Hkv, D, paged):
    """One new token per sequence: empty cache, window shorter and longer than the
    cache, page and tile borders, an idle sequence."""
    c = Case(Hq + D, Hq, Hkv, D, [0, 1, 63, 64, 65, 300, 999, 500], [1, 1, 1, 1, 1, 1, 1, 0], 128, 3, paged=paged)
    c.check(c.run(dreams))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 70), (63, 0), (64, 4), (65, 1), (200, 64), (1000, 5), (2 ** 31 - 1, 0),
                                          (2 ** 31 - 1, 2 ** 31 - 1), (17, 2 ** 31 - 1), (500, 640)])
@pytest.mark.parametrize("kind", ["token", "chunk", "tree"])
def test_windows_and_sinks(dreams, window, sinks, kind):
    n = {"token": [1, 1], "chunk": [150, 37], "tree": [60, 9]}[kind]
    for paged in (False, True):
        c = Case(window % 1000 + sinks % 100, 8, 2, 128, [700, 130], n, window, sinks, tree=kind == "tree", paged=paged)
        c.check(c.run(dreams), n=30)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("T", [2, 17, 64])
def test_trees(dreams, Hq, Hkv, D, T):
    c = Case(T + Hq, Hq, Hkv, D, [0, 400, 61], [T, max(1, T // 2), T], 100, 4, tree=True, paged=T == 17)
    c.check(c.run(dreams), n=40)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("T,L", [(129, 0), (300, 77), (640, 1000)])
def test_prefill(dreams, Hq, Hkv, D, T, L):
    c = Case(T + Hq, Hq, Hkv, D, [L, 0, L // 2], [T, 1, T - 100], 200, 4, paged=T == 300)
    c.check(c.run(dreams), n=40)


@pytest.mark.parametrize("Hq,Hkv,D,B,T,L,window,sinks,tree", [
    (32, 32, 64, 2, 1400, 0, 100, 4, False), (32, 32, 128, 6, 650, 33, 90, 0, False), (32, 8, 128, 40, 64, 200, 150, 3, True),
    (16, 16, 64, 24, 300, 1000, 1, 1, False), (28, 4, 128, 90, 40, 65, 64, 70, True)])
def test_more_blocks_than_the_gpu_holds(dreams, Hq, Hkv, D, B, T, L, window, sinks, tree):
    """Several blocks for every SM, of different lengths, some sequences idle."""
    q_len = [0 if b % 7 == 3 else T - (b * 37) % T for b in range(B)]
    c = Case(B + T, Hq, Hkv, D, [(L * (b + 1)) // B for b in range(B)], q_len, window, sinks, tree=tree, paged=tree, T_max=T)
    c.check(c.run(dreams), n=12)


def test_long_split_lists(dreams):
    """Few heads and a long window: the key list is split over a cluster."""
    c = Case(5, 4, 1, 128, [9001], [1], 8000, 16)
    c.check(c.run(dreams))
    c = Case(6, 2, 2, 64, [5000, 17], [3, 3], 4500, 0, tree=True, paged=True)
    c.check(c.run(dreams))


def test_wide_window_equals_causal_attention(dreams):
    """A window over everything: the rows of dreams_attention's causal mode."""
    c = Case(11, 8, 2, 128, [300, 20], [200, 64], 10 ** 6, 0)
    got = c.run(dreams)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ref, lse, _ = dreams.attention(c.q.cuda(), dreams.KVCache(c.k.cuda(), c.v.cuda()), i32(c.q_len), i32(c.kv_len), c.scale,
                                   dreams.ATTN_CAUSAL, want_lse=True)
    for b in range(2):
        n = c.q_len[b]
        assert (got[0][b, :n].float() - ref[b, :n].float()).abs().max() <= 2.0 ** -7  # |O| < 2: two roundings apart
        assert (got[1][b, :n] - lse[b, :n]).abs().max() <= 1e-4


@pytest.mark.parametrize("kind", ["token", "chunk", "tree"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_slots_do_not_matter(dreams, kind, bad):
    """Slots no query sees hold infinities or NaN, in K and V."""
    n = {"token": [1, 1], "chunk": [90, 200], "tree": [20, 64]}[kind]
    c = Case(21, 8, 2, 128, [500, 333], n, 100, 4, tree=kind == "tree")
    for b in range(2):
        lo, end = c.kv_len[b] - c.window + 1, c.kv_len[b] + n[b]
        for x in (c.k, c.v):
            x[0, b, c.sinks:lo] = bad
            x[0, b, end:] = bad
    c.check(c.run(dreams))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_slot_only_some_rows_see(dreams, bad):
    """V holds an infinity or NaN where some rows of a block see it and others do
    not: only those that do are affected."""
    c = Case(22, 8, 2, 128, [300], [64], 50, 2, tree=True)
    node = 30
    c.v[0, 0, c.kv_len[0] + node, :, 5] = bad
    hit = {(0, t) for t in range(64) if c.kv_len[0] + node in S.visible(t, 300, 50, 2, c.parent[0])}
    assert 0 < len(hit) < 64
    out = c.run(dreams)
    c.check(out, n=600, skip=hit)
    assert not torch.isfinite(out[0][0, [t for _, t in hit], :, 5]).any()
    c = Case(23, 4, 2, 64, [300], [200], 50, 2)
    c.v[0, 0, 290, :, 7] = bad  # leaves the window of query 40
    c.v[0, 0, 450, :, 9] = bad  # enters with query 150, leaves with query 200
    hit = {(0, t) for t in range(200) if t < 40 or t >= 150}
    out = c.run(dreams)
    c.check(out, n=900, skip=hit)
    assert not torch.isfinite(out[0][0, 150:200, :, 9]).any() and not torch.isfinite(out[0][0, :40, :, 7]).any()


def test_large_scores(dreams):
    """Scores of some hundreds: one key takes the whole weight."""
    c = Case(31, 8, 2, 128, [700, 5], [70, 3], 300, 4, kscale=30.0)
    out, lse = c.run(dreams)
    # with dominant scores s the f32 score error is up to 2^-24 D sum|q k| scale, about 1e-2 for |q k| sums of 2000:
    # compare the outputs loosely and the log-sum-exp relatively
    assert torch.isfinite(out[0, :70]).all() and torch.isfinite(lse[0, :70]).all()
    K, V = c.k[0, 0].double().numpy(), c.v[0, 0].double().numpy()
    ref = S.window_rows(c.q[0].double().numpy(), lambda s, g: (K[s, g], V[s, g]), 700, c.scale, 300, 4, lambda h: h // 4,
                        None, [(t, 1) for t in range(70)])
    for t, (o, a, z) in enumerate(ref):
        assert abs(float(lse[0, t, 1]) - z) <= 2e-4 * abs(z)
        assert np.abs(out[0, t, 1].double().cpu().numpy() - o).max() <= 2 * U * np.abs(o).max() + 0.02 * a.max()


def test_strided_queries_layers_streams_and_repeats(dreams):
    """Queries as a view of a fused projection, a cache of three layers, a side
    stream: the same bits as the dense call, every time."""
    c = Case(41, 8, 2, 128, [260, 100, 0], [33, 1, 20], 90, 3, layers=3, layer=2, paged=True)
    a = c.run(dreams)
    c.check(a)
    fused = torch.randn((3, c.T_max, 3, 8, 128), device="cuda").to(torch.bfloat16)
    fused[:, :, 1] = c.q.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for kw in ({"q": fused[:, :, 1]}, {"stream": s}, {}):
        torch.cuda.synchronize()
        r = c.run(dreams, **kw)
        assert torch.equal(a[0], r[0]) and torch.equal(a[1], r[1])


def test_cuda_graph_replay(dreams):
    """A captured call reads lengths and pages at replay: growing by a token."""
    c = Case(42, 8, 2, 128, [300, 40], [1, 1], 64, 2)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    kv, q = dreams.KVCache(c.k.cuda(), c.v.cuda()), c.q.cuda()
    ql, kl = i32(c.q_len), i32(c.kv_len)
    out, lse = torch.empty_like(q), torch.empty((2, 1, 8), device="cuda")
    call = lambda: dreams.window_attention(q, kv, ql, kl, c.scale, 64, 2, out=out, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        kl.copy_(i32([300 + step, 40 + step]))
        graph.replay()
        c.kv_len = [300 + step, 40 + step]
        c.check((out, lse))


def test_cache_beyond_32_bit_offsets(dreams):
    """Pages whose elements start past 2^31 and 2^32."""
    Hkv, D = 8, 128
    pages = (1 << 32) // (64 * Hkv * D) + 40
    k = torch.zeros((pages, 64, Hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    c = Case(51, 32, Hkv, D, [200], [1], 150, 2, paged=True)
    far = torch.tensor([pages - 1 - 3 * i for i in range(c.kp.shape[1])])
    for i in range(c.kp.shape[1]):
        k[far[i]], v[far[i]] = c.kp[0, i].cuda(), c.vp[0, i].cuda()
    table = torch.where(c.table >= 0, far[c.table.clamp(min=0).long()].to(torch.int32), -1).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for T in (1, 64):
        d = Case(51, 32, Hkv, D, [200], [1], 150, 2)
        q = d.q.expand(1, T, 32, D).contiguous() if T > 1 else d.q
        out = torch.full((1, T, 32, D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((1, T, 32), 7.0, device="cuda")
        dreams.window_attention(q.cuda(), dreams.KVCache(k, v, table), i32([1]), i32([200]), d.scale, 150, 2, out=out, lse=lse)
        torch.cuda.synchronize()
        d.k, d.v, d.q, d.T_max = c.k, c.v, q, T
        d.check((out, lse))
    del k, v


def test_data_flags(dreams):
    c = Case(61, 8, 2, 128, [100, 100, 100, 100], [5, 5, 5, 5], 64, 2)
    c.q_len, c.kv_len = [6, -1, 5, 5], [100, 100, -1, c.cap - 4]
    out, lse = c.run(dreams, want=dreams.DATA_BAD_TREE_LEN | dreams.DATA_BAD_KV_LEN)
    assert (out == 7.0).all() and (lse == 7.0).all()
    c = Case(62, 8, 2, 128, [100, 100], [5, 5], 64, 2, tree=True)
    c.parent[1][3] = 3
    out, lse = c.run(dreams, want=dreams.DATA_BAD_PARENT)
    assert (out[1] == 7.0).all() and (out[0] != 7.0).any()
    for entry in (-1, 10 ** 6):
        for T in (5, 70):
            c = Case(63, 8, 2, 128, [300, 300], [T, T], 64, 2, paged=True)
            c.table[1, 4] = entry
            out, lse = c.run(dreams, want=dreams.DATA_BAD_PAGE)
            c.B = 1  # the other sequence is whole
            c.check((out[:1], lse[:1]))


@pytest.mark.parametrize("sinks", [63, 64, 65, 127, 128, 129, 191, 300, 500])
@pytest.mark.parametrize("window,kind", [(50, "chunk"), (129, "chunk"), (64, "tree"), (201, "tree")])
def test_sinks_around_page_ends(dreams, sinks, window, kind):
    """Sinks and window meet inside a tile of two pages, at its end, and overlap."""
    c = Case(3 * sinks + window, 8, 2, 128 if sinks % 2 else 64, [450, 700, 90], [130, 33, 140] if kind == "chunk" else [60, 33, 64], window, sinks,
             tree=kind == "tree", paged=sinks % 3 == 0)
    c.check(c.run(dreams), n=30)


@pytest.mark.parametrize("Hq,Hkv,D", [(28, 4, 128), (16, 1, 64), (32, 8, 128), (20, 10, 64), (32, 32, 128)])
@pytest.mark.parametrize("window", [90, 400, 1100, 2500])
def test_one_sequence_over_clusters(dreams, Hq, Hkv, D, window):
    """A few blocks of one sequence, their tiles split over clusters of every size, some with fewer tiles than CTAs."""
    for T, tree in ((64, True), (70, False)):
        c = Case(Hq + window, Hq, Hkv, D, [2600], [T], window, 3, tree=tree, paged=tree)
        c.check(c.run(dreams), n=40)
