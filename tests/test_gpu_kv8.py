"""GPU parity of kv_quantize (codes and powers bit for bit) and of kv8_attention against
the fp64 oracle on the values that the codes stand for.

Tolerance of the attention, as for windowed attention: probabilities enter the PV
product as bf16 and the output is rounded to bf16 once, each at most u = 2^-8
relative, so with A = sum_j a_j |V_j| an element may be off by u (|O| + A); scores and
sums are f32 (1e-4 of A together for scores of a few units, D products each). The bound is
1.02 u (|O| + A) + 2e-4 A + 1e-6. The log-sum-exp carries the scores' f32 error alone:
1e-4 + 1e-6 |lse|."""
import numpy as np
import pytest
import torch

from oracle import rotary_kv8 as R
from oracle import serving as S

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def codes8(shape, fill=None):
    t = torch.empty(shape, dtype=torch.uint8, device="cuda")
    t.random_(0, 256) if fill is None else t.fill_(fill)
    return t.view(torch.float8_e4m3fn)


def same(a, b):
    return torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)


# ------------------------------------------------------------------ quantize
class Pages:
    """bf16 slots begin .. end - 1 in pages (or a contiguous cache), 8-bit pages of random bytes."""

    def __init__(self, D, Hkv, begin, end, paged=True, layers=2, seed=0, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.B, self.D, self.Hkv, self.begin, self.end, self.layers = len(begin), D, Hkv, begin, end, layers
        self.P = max(1, max(end) // 64 + 1)
        n = self.B * self.P
        shape = (layers, n, 64, Hkv, D) if paged else (layers, self.B, self.P * 64, Hkv, D)
        x = torch.randn((2, *shape), generator=g)
        if scale is not None:  # every page and head of its own size
            x *= torch.exp2(torch.randint(-scale, scale + 1, (2, layers, shape[1], shape[2] // 64, Hkv), generator=g).float()
                            ).repeat_interleave(64, 3)[..., None]
        self.k, self.v = x.to(torch.bfloat16).cuda()
        self.table = torch.randperm(n, generator=g).view(self.B, self.P).to(torch.int32).cuda() if paged else None
        self.table8 = torch.randperm(n + 3, generator=g)[:n].view(self.B, self.P).to(torch.int32).cuda()
        self.k8, self.v8 = codes8((layers, n + 3, 64, Hkv, D)), codes8((layers, n + 3, 64, Hkv, D))
        self.exps = torch.full((layers, n + 3, Hkv, 2), 99, dtype=torch.int16, device="cuda")

    def run(self, dreams, want=0, **kw):
        kv, kv8 = dreams.KVCache(self.k, self.v, self.table), dreams.KV8Cache(self.k8, self.v8, self.exps, self.table8)
        st = i32([0])
        new = dreams.kv_quantize(kv, kv8, i32(self.begin), i32(self.end), status=st, **kw)
        torch.cuda.synchronize()
        assert int(st) == want
        return new.tolist()

    def rows(self, x, l, b, e):
        if self.table is None:
            return x[l, b, 64 * e:64 * e + 64]
        return x[l, int(self.table[b, e])]

    def want(self, skip=()):
        """The 8-bit arrays after the call, from copies of what they were."""
        k8, v8, exps = (t.cpu() for t in (self.k8.view(torch.uint8), self.v8.view(torch.uint8), self.exps))
        for b in range(self.B):
            for e in range(self.begin[b] // 64, self.end[b] // 64):
                if (b, e) in skip:
                    continue
                for l in range(self.layers):
                    z = int(self.table8[b, e])
                    for i, (x, y) in enumerate(((self.k, k8), (self.v, v8))):
                        c, es = R.quantize_page(self.rows(x, l, b, e).double().cpu().numpy())
                        y[l, z], exps[l, z, :, i] = torch.tensor(c), torch.tensor(es)
        return k8, v8, exps

    def check(self, want):
        assert torch.equal(self.exps.cpu(), want[2])
        for got, w in ((self.k8, want[0]), (self.v8, want[1])):
            g = got.view(torch.uint8).cpu()
            assert torch.equal(g, w), int((g != w).sum())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("paged", [True, False])
def test_quantize(dreams, D, paged):
    """No page, one, several; lengths around page ends; everything else untouched."""
    c = Pages(D, 3, [0, 0, 0, 64, 128, 64, 0], [0, 63, 64, 64, 300, 191, 257], paged, scale=6)
    w = c.want()
    assert c.run(dreams) == [0, 0, 64, 64, 256, 128, 256]
    c.check(w)


def test_quantize_extremes(dreams):
    """The ends of the range of powers, largest magnitudes on both sides of 1.75 2^n, ties, zeros of both signs, subnormals."""
    c = Pages(64, 4, [0], [256], layers=1)
    for pg, head, amax in ((0, 0, 1.75), (0, 1, 1.7578125), (0, 2, 448.0), (0, 3, 1.9921875), (1, 0, 3.38e38), (1, 1, 2.0 ** 120), (1, 2, 2.0 ** -87),
                           (1, 3, 2.0 ** -100), (2, 0, 0.0), (2, 1, 2.0 ** -126), (2, 2, 2.0 ** -133), (2, 3, 1.75 * 2.0 ** 127)):
        x = c.rows(c.k, 0, 0, pg)[:, head]
        x.copy_((torch.rand_like(x.float()) * 2 - 1) * amax)
        x[5, 7] = -amax
        x[6, 8], x[6, 9] = -0.0, 0.0
    t = torch.tensor(R.values()[:118])  # (up to 255 they and the values between two are bf16)
    ties = ((t[1:] + t[:-1]) / 2).float()
    x = c.rows(c.v, 0, 0, 3)[:, 0]
    x.zero_()
    x.view(64, 64)[:2].copy_(torch.cat([ties, -ties[:11]]).view(2, 64))
    x[9, 9] = 448.0
    w = c.want()
    assert c.run(dreams) == [256]
    c.check(w)


def test_quantize_not_finite(dreams):
    c = Pages(128, 2, [0], [192], layers=2)
    c.rows(c.k, 1, 0, 0)[3, 1, 5] = float("nan")
    c.rows(c.v, 0, 0, 2)[63, 0, 127] = float("-inf")
    keep = c.want()[2]
    assert c.run(dreams) == [192]
    assert torch.equal(c.exps.cpu(), keep)
    z = c.table8[0].tolist()
    assert int(c.exps[1, z[0], 1, 0]) == int(c.exps[0, z[2], 0, 1]) == dreams.KV8_NOT_FINITE == R.NOT_FINITE
    assert int((c.exps == dreams.KV8_NOT_FINITE).sum()) == 2


def test_quantize_bad_data(dreams):
    """Bad lengths skip their sequence; a page missing on either side is skipped and ends the new length."""
    begin, end = [-64, 32, 128, 0, 0, 0, 64], [64, 128, 64, 10 ** 6, 320, 256, 200]
    c = Pages(64, 2, begin[:3] + [0] * 3 + [64], [0, 0, 0, 0, 320, 256, 200])
    c.begin, c.end = begin, [e if e < 1000 else 0 for e in end]
    skip = {(b, e) for b in range(3) for e in range(-2, 9)} | {(4, 2), (5, 0)}
    c.table[4, 2], c.table8[5, 0] = -1, c.k8.shape[1]
    w = c.want(skip)
    c.end = end
    assert c.run(dreams, dreams.DATA_BAD_KV_LEN | dreams.DATA_BAD_PAGE) == [-64, 32, 128, 0, 128, 0, 192]
    c.check(w)


def test_quantize_many_sequences(dreams):
    """More sequences than a block's threads; captured and replayed."""
    B = 300
    c = Pages(64, 1, [64 * (b % 3) for b in range(B)], [64 * (b % 3) + (b * 37) % 190 for b in range(B)], layers=1)
    w = c.want()
    lens = [x + n // 64 * 64 for x, n in zip(c.begin, [(b * 37) % 190 for b in range(B)])]
    assert c.run(dreams) == lens
    c.check(w)
    kv, kv8 = dreams.KVCache(c.k, c.v, c.table), dreams.KV8Cache(c.k8, c.v8, c.exps, c.table8)
    bg, en, new = i32(c.begin), i32(c.end), i32([0] * B)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dreams.kv_quantize(kv, kv8, bg, en, new_len8=new)
    c.k.normal_()
    c.v.mul_(3)
    w = c.want()
    graph.replay()
    assert new.tolist() == lens
    c.check(w)


# ------------------------------------------------------------------ attention
def _tree(rng, T, T_max):
    par = [-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, T)]
    return (par + [-1] * T_max)[:T_max]


class Case:
    """One seeded problem: all slots' values in fp64 (those below len8 as their codes give them), both caches' pages in
    random order, everything that no query may see filled with NaN or without a page."""

    def __init__(self, seed, Hq, Hkv, D, kv_len, q_len, len8, window=2 ** 31 - 1, sinks=0, tree=False, paged=True, T_max=None, layers=1, layer=0,
                 kscale=1.0, spread=1, mark=None):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.D, self.layer, self.scale = len(kv_len), Hq, Hkv, D, layer, D ** -0.5
        self.kv_len, self.q_len, self.len8, self.window, self.sinks = kv_len, q_len, len8, window, sinks
        self.T_max = T_max or max(1, max(q_len))
        self.P = max(L + n for L, n in zip(kv_len, q_len)) // 64 + 1
        cap = self.P * 64
        self.parent = [_tree(rng, max(1, n), self.T_max) for n in q_len] if tree else None
        self.q = torch.randn((self.B, self.T_max, Hq, D), generator=g).to(torch.bfloat16)
        kv = torch.randn((2, layers, self.B, cap, Hkv, D), generator=g)
        kv[0] *= kscale
        size = torch.randint(-spread, spread + 1, (layers, self.B, self.P, Hkv), generator=g).float()
        kv[1] *= torch.exp2(size).repeat_interleave(64, 2)[..., None]  # V's pages differ in size
        kv = kv.to(torch.bfloat16)
        seen = lambda b, e: e * 64 < kv_len[b] + q_len[b] and (64 * e + 64 > kv_len[b] - window + 1 or 64 * e < sinks)  # noqa: E731
        use8 = [(b, e) for b in range(self.B) for e in range(self.P) if seen(b, e) and e * 64 < len8[b]]
        use = [(b, e) for b in range(self.B) for e in range(self.P) if seen(b, e) and e * 64 >= len8[b]]
        n8, n = len(use8) + 2, len(use) + 2
        self.k8, self.v8 = (torch.randint(0, 256, (layers, n8, 64, Hkv, D), generator=g, dtype=torch.uint8) for _ in range(2))
        self.exps = torch.full((layers, n8, Hkv, 2), 119, dtype=torch.int16)
        self.table8, self.table = (torch.full((self.B, self.P), -1, dtype=torch.int32) for _ in range(2))
        ids8, ids = rng.permutation(n8), rng.permutation(n)
        self.vals = kv.double().numpy()
        for i, (b, e) in enumerate(use8):
            z = int(ids8[i])
            self.table8[b, e] = z
            for l in range(layers):
                for j, x8 in ((0, self.k8), (1, self.v8)):
                    c, es = R.quantize_page(self.vals[j, l, b, 64 * e:64 * e + 64])
                    if mark and (b, e, j) in mark:
                        es[:] = R.NOT_FINITE
                    x8[l, z], self.exps[l, z, :, j] = torch.tensor(c), torch.tensor(es)
                    self.vals[j, l, b, 64 * e:64 * e + 64] = R.decode(c, es[None, :, None])
        if paged:
            self.k, self.v = (torch.full((layers, n, 64, Hkv, D), float("nan"), dtype=torch.bfloat16) for _ in range(2))
            for i, (b, e) in enumerate(use):
                z = int(ids[i])
                self.table[b, e] = z
                m = max(0, min(64, kv_len[b] + q_len[b] - 64 * e))  # (what lies behind the last row is NaN)
                self.k[:, z, :m], self.v[:, z, :m] = kv[0, :, b, 64 * e:64 * e + m], kv[1, :, b, 64 * e:64 * e + m]
        else:
            self.table = None
            self.k, self.v = kv[0].clone(), kv[1].clone()
            for b in range(self.B):
                for x in (self.k, self.v):
                    x[:, b, :len8[b]] = x[:, b, kv_len[b] + q_len[b]:] = float("nan")

    def run(self, dreams, want=0, q=None, **kw):
        kv = dreams.KVCache(self.k.cuda(), self.v.cuda(), None if self.table is None else self.table.cuda())
        kv8 = dreams.KV8Cache(*(x.cuda().view(torch.float8_e4m3fn) for x in (self.k8, self.v8)), self.exps.cuda(), self.table8.cuda())
        st = i32([0])
        out = torch.full((self.B, self.T_max, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.B, self.T_max, self.Hq), 7.0, dtype=torch.float32, device="cuda")
        dreams.kv8_attention(self.q.cuda() if q is None else q, kv8, kv, i32(self.q_len), i32(self.kv_len), i32(self.len8), self.scale,
                             window=self.window, sinks=self.sinks, parent=None if self.parent is None else i32(self.parent), layer=self.layer,
                             out=out, lse=lse, status=st, **kw)
        torch.cuda.synchronize()
        assert int(st) == want
        return out, lse

    def check(self, got, n=40, seed=0, skip=(), nan=None, cut=None):
        """nan: whether a row (b, t) has to be NaN; cut: slots that read as zeros."""
        out, lse = got[0].float().cpu().numpy().astype(np.float64), got[1].cpu().numpy().astype(np.float64)
        rng = np.random.default_rng(seed)
        G = self.Hq // self.Hkv
        for b in range(self.B):
            assert (out[b, self.q_len[b]:] == 7.0).all() and (lse[b, self.q_len[b]:] == 7.0).all()
            if b in skip:
                assert (out[b] == 7.0).all() and (lse[b] == 7.0).all()
                continue
            sel = [(t, h) for t in range(self.q_len[b]) for h in range(self.Hq)]
            if len(sel) > n:  # the ends and some between
                sel = [sel[0], sel[-1]] + [sel[i] for i in rng.choice(len(sel), n, replace=False)]
            K, V = (x[self.layer, b].copy() for x in self.vals)
            for s in cut or ():
                K[s] = V[s] = 0.0
            par = None if self.parent is None else self.parent[b]
            ref = S.window_rows(self.q[b].double().numpy(), lambda s, g: (K[s, g], V[s, g]), self.kv_len[b], self.scale, self.window,
                                self.sinks, lambda h: h // G, par, sel)
            for (t, h), (o, a, z) in zip(sel, ref):
                if nan is not None and nan(b, t):
                    assert np.isnan(out[b, t, h]).all(), (b, t, h)
                    continue
                err = np.abs(out[b, t, h] - o)
                tol = 1.02 * U * (np.abs(o) + a) + 2e-4 * a + 1e-6
                assert (err <= tol).all(), (b, t, h, float((err / tol).max()))
                assert abs(lse[b, t, h] - z) <= 1e-4 + 1e-6 * abs(z), (b, t, h, lse[b, t, h], z)


HEADS = [(28, 4, 128), (32, 8, 128), (8, 8, 128), (4, 4, 64), (16, 1, 64), (10, 2, 128), (128, 1, 128)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("paged", [True, False])
def test_single_tokens(dreams, Hq, Hkv, D, paged):
    """One new token: empty caches, all of the prefix in 8 bits or none, lengths around page ends, an idle sequence."""
    c = Case(Hq + D, Hq, Hkv, D, [0, 1, 63, 64, 65, 300, 999, 500, 128, 700], [1, 1, 1, 1, 1, 1, 1, 0, 1, 1], [0, 0, 0, 64, 64, 128, 960, 448, 0, 640],
             paged=paged)
    c.check(c.run(dreams))


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("kind", ["few", "chunk", "tree"])
def test_rows(dreams, Hq, Hkv, D, kind):
    n = {"few": [2, 3, 1, 2], "chunk": [150, 37, 1, 0], "tree": [60, 9, 1, 33]}[kind]
    c = Case(Hq + D + len(kind), Hq, Hkv, D, [700, 130, 64, 257], n, [640, 64, 64, 192], tree=kind == "tree")
    c.check(c.run(dreams), n=25)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 70), (63, 0), (64, 4), (65, 1), (200, 64), (200, 100), (1000, 5), (2 ** 31 - 1, 2 ** 31 - 1),
                                          (17, 2 ** 31 - 1), (300, 640)])
@pytest.mark.parametrize("kind", ["token", "chunk", "tree"])
def test_windows_and_sinks(dreams, window, sinks, kind):
    """What the window leaves out has no page in either cache; sinks and window in 8 bits, in bf16, and across."""
    n = {"token": [1, 1, 1], "chunk": [150, 37, 20], "tree": [60, 9, 30]}[kind]
    for len8 in ([640, 128, 0], [64, 64, 0], [192, 0, 0]):
        c = Case(window % 1000 + sinks % 100, 8, 2, 128, [700, 130, 70], n, len8, window, sinks, tree=kind == "tree")
        c.check(c.run(dreams), n=20)


@pytest.mark.parametrize("T,kv", [(1, 3000), (2, 3000), (9, 3000), (64, 4100), (300, 2500)])
@pytest.mark.parametrize("D", [64, 128])
def test_long_caches(dreams, T, kv, D):
    """Lists split over CTAs, one and several sequences."""
    for B in (1, 3):
        c = Case(T + D + B, 8, 2, D, [kv - 777 * b for b in range(B)], [T] * B, [(kv - 777 * b) // 64 * 64 - 64 * b for b in range(B)])
        c.check(c.run(dreams), n=15)


@pytest.mark.parametrize("T", [1, 3, 40])
def test_pages_of_very_different_size(dreams, T):
    """V's pages differ by 2^80: what a row hardly looks at does not drown what it looks at, nor the other way round."""
    c = Case(T, 8, 2, 128, [400], [T], [384], spread=40)
    got = c.run(dreams)
    out = got[0].float().cpu().numpy().astype(np.float64)
    K, V = (x[0, 0] for x in c.vals)
    sel = [(t, h) for t in range(T) for h in range(8)][:40]
    ref = S.window_rows(c.q[0].double().numpy(), lambda s, g: (K[s, g], V[s, g]), 400, c.scale, c.window, 0, lambda h: h // 4, None, sel)
    for (t, h), (o, a, z) in zip(sel, ref):
        assert (np.abs(out[0, t, h] - o) <= 1.02 * U * (np.abs(o) + a) + 2e-4 * a).all()


@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("kscale", [8.0, 100.0])
def test_dominated_softmax(dreams, T, kscale):
    """Scores of some hundreds: a row's few largest decide, and they come late. f32 scores of magnitude x are off by some
    2^-22 x, so weights by that share: the bound of the scores' part grows with kscale."""
    c = Case(T + 5, 8, 2, 128, [700], [T], [640], kscale=kscale)
    got = c.run(dreams)
    out, lse = got[0].float().cpu().numpy().astype(np.float64), got[1].cpu().numpy()
    K, V = (x[0, 0] for x in c.vals)
    sel = [(t, h) for t in range(T) for h in range(8)][-40:]
    ref = S.window_rows(c.q[0].double().numpy(), lambda s, g: (K[s, g], V[s, g]), 700, c.scale, c.window, 0, lambda h: h // 4, None, sel)
    for (t, h), (o, a, z) in zip(sel, ref):
        # D products of up to 4 units x kscale, rounded in f32 along their sum of up to 128 terms: 2^-24 D^(1/2) of their
        # magnitudes' sum, 128 x 0.7 kscale / 11 = 8 kscale, and twice that for both ends of a difference
        e = 2 * 8 * kscale * 128 * 2.0 ** -24
        assert (np.abs(out[0, t, h] - o) <= 1.02 * U * (np.abs(o) + a) + (2e-4 + 2 * e) * a + 1e-6).all()
        assert abs(lse[0, t, h] - z) <= 1e-4 + 1e-6 * abs(z) + e


@pytest.mark.parametrize("T", [1, 40])
def test_largest_values(dreams, T):
    """K and V at the top of what pages may hold for finite results: powers above 7."""
    c = Case(T, 4, 2, 64, [200], [T], [192])
    up = 40  # V times 2^40
    c.exps[:, :, :, 1] = torch.where(c.exps[:, :, :, 1] == 119, 119, c.exps[:, :, :, 1] + up)
    c.vals[1, 0, 0, :192] *= 2.0 ** up
    c.v = (c.v.float() * 2.0 ** up).to(torch.bfloat16)
    c.vals[1, 0, 0, 192:] *= 2.0 ** up
    c.check(c.run(dreams))


@pytest.mark.parametrize("T", [1, 4, 70])
@pytest.mark.parametrize("j", [0, 1])
def test_pages_that_were_not_finite(dreams, T, j):
    """Rows that see a marked page are NaN; rows whose window has passed it, in the same block, are not."""
    window = 2 ** 31 - 1 if T == 1 else 100
    c = Case(T, 8, 2, 128, [300, 300], [T, T], [256, 256], window, mark={(0, 3, j)})
    last = 255  # of page 3
    c.check(c.run(dreams), nan=lambda b, t: b == 0 and 300 + t - last < window)


@pytest.mark.parametrize("T", [1, 4, 9, 70])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("j", [0, 1])
def test_what_was_not_finite_before(dreams, T, bad, j):
    """The same through kv_quantize, whose codes of such values stand for nothing."""
    window = 2 ** 31 - 1 if T == 1 else 100
    c = Case(T, 8, 2, 128, [300, 300], [T, T], [256, 256], window)
    z, bf = int(c.table8[0, 3]), torch.randn((1, 1, 64, 2, 128)).to(torch.bfloat16)
    k, v = bf.clone(), bf.clone()
    (k, v)[j][0, 0, 60] = bad
    one = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
    one[0, 3] = 0
    kv8 = dreams.KV8Cache(codes8((1, 1, 64, 2, 128)), codes8((1, 1, 64, 2, 128)), torch.zeros((1, 1, 2, 2), dtype=torch.int16, device="cuda"), one)
    assert dreams.kv_quantize(dreams.KVCache(k.cuda(), v.cuda(), one), kv8, i32([192]), i32([256])).tolist() == [256]
    c.k8[:, z], c.v8[:, z], c.exps[:, z] = kv8.k[:, 0].view(torch.uint8).cpu(), kv8.v[:, 0].view(torch.uint8).cpu(), kv8.exps[:, 0].cpu()
    assert (c.exps[0, z, :, j] == R.NOT_FINITE).all() and (c.exps[0, z, :, 1 - j] < 0).all()
    for x, y, e in ((c.vals[0], c.k8, c.exps[:, :, :, 0]), (c.vals[1], c.v8, c.exps[:, :, :, 1])):
        x[0, 0, 192:256] = R.decode(y[0, z].numpy(), e[0, z].numpy()[None, :, None])
    c.check(c.run(dreams), nan=lambda b, t: b == 0 and 300 + t - 255 < window)


@pytest.mark.parametrize("T", [1, 40])
def test_missing_pages_read_as_zeros(dreams, T):
    for table, e in (("table8", 1), ("table8", 3), ("table", 4), ("table", 5)):
        c = Case(T, 8, 2, 128, [330], [T], [256])
        getattr(c, table)[0, e] = 10 ** 6 if e % 2 else -1
        if e * 64 >= 330 + T:
            continue
        c.check(c.run(dreams, dreams.DATA_BAD_PAGE), cut=range(64 * e, min(64 * e + 64, 330 + T)))


@pytest.mark.parametrize("T", [1, 40])
def test_bad_data(dreams, T):
    """Bad sequences are flagged and left untouched, the others computed."""
    for kw, want in ((dict(len8=[32, 128]), dreams.DATA_BAD_KV_LEN), (dict(len8=[-64, 128]), dreams.DATA_BAD_KV_LEN), (dict(len8=[320, 128]), dreams.DATA_BAD_KV_LEN),
                     (dict(kv_len=[-1, 130]), dreams.DATA_BAD_KV_LEN), (dict(len8=[2 ** 31 - 64, 128]), dreams.DATA_BAD_KV_LEN), (dict(kv_len=[10 ** 6, 130]), dreams.DATA_BAD_KV_LEN),
                     (dict(q_len=[-1, T]), dreams.DATA_BAD_TREE_LEN), (dict(q_len=[T + 1, T]), dreams.DATA_BAD_TREE_LEN)):
        c = Case(T, 8, 2, 128, [300, 130], [T, T], [256, 128])
        for k, v in kw.items():
            setattr(c, k, v)
        got = c.run(dreams, want)
        c.q_len = [0, T]
        c.check(got, skip=(0,))
    if T > 1:
        c = Case(T, 8, 2, 128, [300, 130], [T, T], [256, 128], tree=True)
        c.parent[0][5] = 5
        c.check(c.run(dreams, dreams.DATA_BAD_PARENT), skip=(0,))


def test_a_short_table_of_8_bit_pages(dreams):
    """The 8-bit cache may have fewer entries to a sequence than the bf16 one; beyond them len8 is bad."""
    c = Case(1, 8, 2, 128, [700, 400], [1, 1], [128, 128])
    c.table8 = c.table8[:, :2].contiguous()
    c.check(c.run(dreams))
    c.len8 = [192, 128]
    c.check(c.run(dreams, dreams.DATA_BAD_KV_LEN), skip=(0,))


def test_infinities_in_new_rows_stay_with_those_who_see_them(dreams):
    """A tree's node with an infinity or a NaN in V: rows off its path keep their values."""
    for bad in (float("inf"), float("nan")):
        for T, heads in ((16, (2, 2)), (60, (8, 2))):
            c = Case(T, *heads, 128, [300], [T], [256], tree=True)
            c.parent[0] = [-1] + [0] * (T - 1)
            page, row = divmod(300 + 7, 64)
            z = int(c.table[0, page])
            c.v[0, z, row] = bad
            clean = c.vals[1].copy()
            got = c.run(dreams)
            assert not torch.isfinite(got[0][0, 7].float()).any()
            got[0][0, 7] = 0
            c.vals[1] = clean
            keep = [t for t in range(T) if t != 7]
            ref = S.window_rows(c.q[0].double().numpy(), lambda s, g: (c.vals[0][0, 0][s, g], clean[0, 0][s, g]), 300, c.scale, c.window, 0,
                                lambda h: h // (heads[0] // heads[1]), c.parent[0], [(t, 0) for t in keep])
            for t, (o, a, z) in zip(keep, ref):
                assert (np.abs(got[0][0, t, 0].double().cpu().numpy() - o) <= 1.02 * U * (np.abs(o) + a) + 2e-4 * a + 1e-6).all()


def test_layers_strides_and_repeats(dreams):
    """Another layer than the first, Q as a view of a fused projection, the same call twice."""
    for T in (1, 50):
        c = Case(T + 1, 8, 2, 64, [333, 80], [T, T], [320, 64], layers=3, layer=2)
        a = c.run(dreams)
        c.check(a)
        fused = torch.randn((2, T, 3, 8, 64), device="cuda").to(torch.bfloat16)
        fused[:, :, 1] = c.q.cuda()
        b = c.run(dreams, q=fused[:, :, 1])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_agrees_with_windowed_attention_on_the_same_values(dreams):
    """With nothing in 8 bits the two calls compute the same thing; and so they do on a bf16 cache of the stored values."""
    for T, tree in ((1, False), (60, True), (200, False)):
        c = Case(T, 8, 2, 128, [500], [T], [0], tree=tree)
        a = c.run(dreams)
        kv = dreams.KVCache(c.k.cuda(), c.v.cuda(), c.table.cuda())
        par = None if c.parent is None else i32(c.parent)
        b = dreams.window_attention(c.q.cuda(), kv, i32([T]), i32([500]), c.scale, 2 ** 31 - 1, parent=par, want_lse=True)
        assert (a[0].float() - b[0].float()).abs().max() <= 2 * U * b[0].float().abs().max() and (a[1] - b[1]).abs().max() < 1e-4


def test_streams_and_graphs(dreams):
    for T in (1, 60):
        c = Case(T + 3, 8, 2, 128, [500, 90], [T, T], [448, 64], tree=T > 1)
        want = c.run(dreams)
        kv = dreams.KVCache(c.k.cuda(), c.v.cuda(), c.table.cuda())
        kv8 = dreams.KV8Cache(*(x.cuda().view(torch.float8_e4m3fn) for x in (c.k8, c.v8)), c.exps.cuda(), c.table8.cuda())
        par = None if c.parent is None else i32(c.parent)
        ql, kl, l8 = i32(c.q_len), i32(c.kv_len), i32(c.len8)
        side, q = torch.cuda.Stream(), torch.zeros_like(c.q, device="cuda")
        src = c.q.cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            busy = torch.randn((4096, 4096), device="cuda")
            for _ in range(20):
                busy = busy @ busy
                busy = busy / busy.norm()
            q.copy_(src)
        out, lse = dreams.kv8_attention(q, kv8, kv, ql, kl, l8, c.scale, parent=par, want_lse=True, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = dreams.kv8_attention(q, kv8, kv, ql, kl, l8, c.scale, parent=par, want_lse=True)
        q.zero_()
        graph.replay()
        q.copy_(src)
        graph.replay()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
