"""GPU parity of rope and kv_append_rope against the fp64 oracle.

Tolerance, for a pair (u, v) and S = factor (|u| + |v|). The angle's 32 bits are cut
off by 2 pi 2^-32 and rounded to f32 (2^-24 of at most pi: 1.9e-7), sincospif is within
two units of 2^-24 (1.2e-7), the factor, the two products and their sum round by 2^-24
each (1.8e-7): 5e-7 S altogether. A bf16 result adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import rotary_kv8 as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(got, x, phases, pos, layout, factor=1.0, transpose=False):
    """Rows got, x [N, H, D] at positions pos [N] (or [N, n_pairs])."""
    g, x = got.double().cpu().numpy(), x.double().cpu().numpy()
    n = len(phases)
    for i in range(len(x)):
        want = R.rotate(x[i], phases, pos[i], layout, factor, transpose)
        tol = np.zeros_like(want)
        for a, b in R.pairs(n, layout):
            tol[:, a] = tol[:, b] = 5e-7 * abs(factor) * (np.abs(x[i, :, a]) + np.abs(x[i, :, b])) + 1e-38
        if got.dtype == torch.bfloat16:
            tol += np.where(tol > 0, 2.0 ** -8 * np.abs(want), 0)
        err = np.abs(g[i] - want)
        assert (err <= tol).all(), (i, pos[i], float(err.max()))


def phases_of(r):
    return [p % 2 ** 64 for p in r.phase.tolist()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(128, 128), (64, 64), (128, 96), (64, 48), (128, 58), (64, 10), (80, 80), (96, 32), (6, 2), (2, 2), (34, 34), (512, 512), (512, 510),
                                   (256, 2)])
def test_shapes(dreams, dtype, layout, D, rot):
    g = torch.Generator().manual_seed(D + rot)
    r = dreams.Rotary.make(rot, layout=layout, gain=1.25)
    for B, T, H in ((1, 1, 1), (2, 7, 3), (3, 1, 28), (1, 33, 9)):
        x = torch.randn((B, T, H, D), generator=g).to(dtype).cuda()
        start = i32([5, 0, 70000][:B])
        y = dreams.rope(x, r, start=start)
        z = dreams.rope(x, r, start=start, transpose=True)
        pos = [int(s) + t for s in start.tolist() for t in range(T)]
        check(y.flatten(0, 1), x.flatten(0, 1), phases_of(r), pos, layout, r.factor)
        check(z.flatten(0, 1), x.flatten(0, 1), phases_of(r), pos, layout, r.factor, True)
    assert torch.equal(y[..., rot:], x[..., rot:])


def test_many_tokens(dreams):
    """Several tokens to a block, ragged at the end, heads that are no multiple of a turn."""
    r = dreams.Rotary.make(128)
    for B, T, H in ((2, 1001, 5), (1, 700, 41), (5, 333, 1)):
        x = torch.randn((B, T, H, 128), device="cuda").to(torch.bfloat16)
        y = dreams.rope(x, r)
        for t in (0, 1, 2, 3, T // 2, T - 2, T - 1):
            check(y[:, t], x[:, t], phases_of(r), [t] * B, "half")
        assert torch.equal(y, dreams.rope(x, r, positions=torch.arange(T, dtype=torch.int32, device="cuda").expand(B, T).contiguous()))


def test_far_and_negative_positions(dreams):
    """One integer product gives the angle: as exact at 2^31 as at 1."""
    r = dreams.Rotary.make(64)
    pos = [0, 1, -1, 10 ** 6, -10 ** 6, 2 ** 31 - 1, -2 ** 31, 123456789]
    x = torch.randn((1, len(pos), 2, 64), device="cuda")
    check(dreams.rope(x, r, positions=i32([pos]))[0], x[0], phases_of(r), pos, "half")
    assert torch.equal(dreams.rope(x, r, start=i32([7])), dreams.rope(x, r, positions=i32([[7 + t for t in range(len(pos))]])))
    for start in (2 ** 31 - 3, -2 ** 31, -4):  # (tokens past 2^31 go on from it)
        check(dreams.rope(x, r, start=i32([start]))[0], x[0], phases_of(r), [start + t for t in range(len(pos))], "half")


def test_axes(dreams):
    r = dreams.Rotary.make(16, axis=[0, 0, 1, 1, 1, 2, 2, 0], layout="interleaved")
    pos = torch.randint(0, 3000, (3, 2, 5), dtype=torch.int32)
    x = torch.randn((2, 5, 3, 64), device="cuda").to(torch.bfloat16)
    y = dreams.rope(x, r, positions=pos.cuda())
    per_pair = pos[torch.tensor([0, 0, 1, 1, 1, 2, 2, 0])].permute(1, 2, 0).flatten(0, 1).tolist()
    check(y.flatten(0, 1), x.flatten(0, 1), phases_of(r), per_pair, "interleaved")
    # an axis that the call does not have is flagged and counts as the first
    st = i32([0])
    z = dreams.rope(x, r, positions=pos[:2].contiguous().cuda(), status=st)
    assert int(st) == dreams.DATA_BAD_INDEX
    first = pos[torch.tensor([0, 0, 1, 1, 1, 0, 0, 0])].permute(1, 2, 0).flatten(0, 1).tolist()
    check(z.flatten(0, 1), x.flatten(0, 1), phases_of(r), first, "interleaved")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_strides(dreams, layout):
    """Views of a fused projection, head-major tensors, odd offsets, broadcast inputs, in place."""
    r = dreams.Rotary.make(64, layout=layout)
    s = i32([3, 9])
    big = torch.randn((2, 6, 3, 4, 64), device="cuda").to(torch.bfloat16)
    dense = lambda x: dreams.rope(x.contiguous(), r, start=s)  # noqa: E731
    v = big[:, :, 1]
    assert torch.equal(dreams.rope(v, r, start=s), dense(v))
    hm = torch.randn((2, 4, 6, 64), device="cuda").transpose(1, 2)
    out = torch.empty((2, 4, 6, 64), device="cuda").transpose(1, 2)
    assert torch.equal(dreams.rope(hm, r, start=s, out=out), dense(hm)) and out.stride() == hm.stride()
    odd = torch.randn(2 * 6 * 4 * 67 + 1, device="cuda").to(torch.bfloat16)[1:].as_strided((2, 6, 4, 64), (6 * 4 * 67, 4 * 67, 67, 1))
    assert torch.equal(dreams.rope(odd, r, start=s), dense(odd))
    one = torch.randn((2, 1, 1, 64), device="cuda").expand(2, 6, 4, 64)
    assert torch.equal(dreams.rope(one, r, start=s), dense(one))
    rest = big[:, :, 0].clone(), big[:, :, 2].clone()
    want = dense(v)
    assert dreams.rope(v, r, start=s, out=v) is v and torch.equal(v, want)
    assert torch.equal(big[:, :, 0], rest[0]) and torch.equal(big[:, :, 2], rest[1])
    with pytest.raises(dreams.DreamsError):
        dreams.rope(one.contiguous(), r, start=s, out=torch.empty((2, 1, 1, 64), device="cuda").expand(2, 6, 4, 64))


def test_values_that_are_not_finite_stay_in_their_pair(dreams):
    r = dreams.Rotary.make(32)
    for rot_layout in ("half", "interleaved"):
        r = dreams.Rotary.make(32, layout=rot_layout)
        x = torch.randn((1, 4, 2, 64), device="cuda").to(torch.bfloat16)
        x[0, 1, 0, 3], x[0, 2, 1, 40] = float("nan"), float("inf")
        y = dreams.rope(x, r)
        a, b = (3, 19) if rot_layout == "half" else (2, 3)
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[0, 1, 0, a] = bad[0, 1, 0, b] = True
        assert torch.equal(torch.isnan(y), bad) and y[0, 2, 1, 40] == float("inf")


def test_gradient_of_a_loss(dreams):
    """The transposed map against differences of the loss sum(w * rope(x))."""
    r = dreams.Rotary.make(8, gain=1.5)
    x, w = torch.randn((1, 3, 2, 12), device="cuda"), torch.randn((1, 3, 2, 12), device="cuda")
    s = i32([1000])
    grad = dreams.rope(w, r, start=s, transpose=True)
    loss = lambda y: (dreams.rope(y, r, start=s).double() * w.double()).sum().item()  # noqa: E731
    for i in range(0, x.numel(), 5):
        d = torch.zeros_like(x)
        d.view(-1)[i] = 0.5
        # f32 outputs of some units, each off by a few 2^-24 of them, over a step of one
        assert abs(loss(x + d) - loss(x - d) - grad.view(-1)[i].item()) < 1e-5


class Rows:
    """Q, K and V rows as views of one projection, and a cache whose other bytes are known."""

    def __init__(self, Hq, Hkv, D, kv_len, n_new, paged, T_max=None, layers=2, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.T = len(kv_len), T_max or max(n_new)
        self.Hq, self.Hkv, self.D, self.kv_len, self.n_new = Hq, Hkv, D, kv_len, n_new
        self.P = (max(kv_len) + self.T) // 64 + 1
        qkv = torch.randn((self.B, self.T, Hq + 2 * Hkv, D), generator=g).to(torch.bfloat16).cuda()
        self.q, self.k, self.v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        n = self.B * self.P
        shape = (layers, n + 2, 64, Hkv, D) if paged else (layers, self.B, self.P * 64, Hkv, D)
        self.kc, self.vc = (torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        self.table = torch.randperm(n + 2, generator=g)[:n].view(self.B, self.P).to(torch.int32).cuda() if paged else None

    def cache(self, dreams):
        return dreams.KVCache(self.kc, self.vc, self.table)

    def place(self, b, s):
        return (int(self.table[b, s // 64]), s % 64) if self.table is not None else (b, s)


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("layout,D,rot", [("half", 128, 128), ("interleaved", 64, 64), ("half", 64, 32), ("half", 128, 58), ("interleaved", 128, 58), ("half", 8, 8),
                                          ("half", 24, 16)])
def test_append(dreams, paged, layout, D, rot):
    """Slots around page ends, an idle sequence, rows past n_new, everything else untouched."""
    c = Rows(6, 2, D, [0, 63, 64, 200, 130], [5, 3, 1, 0, 70], paged, seed=D + rot)
    r = dreams.Rotary.make(rot, layout=layout)
    kv, before = c.cache(dreams), (c.kc.clone(), c.vc.clone())
    qo = torch.full((c.B, c.T, c.Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    st = i32([0])
    assert dreams.kv_append_rope(kv, c.k, c.v, r, i32(c.kv_len), i32(c.n_new), q=c.q, q_out=qo, layer=1, status=st) is qo and int(st) == 0
    want_k, want_v = before[0].clone(), before[1].clone()
    for b in range(c.B):
        n = c.n_new[b]
        assert (qo[b, n:] == 7.0).all()
        pos = [c.kv_len[b] + t for t in range(n)]
        if n:
            check(qo[b, :n], c.q[b, :n], phases_of(r), pos, layout)
            rows = torch.stack([c.kc[1][c.place(b, p)] for p in pos])
            check(rows, c.k[b, :n], phases_of(r), pos, layout)
        for t, p in enumerate(pos):
            want_k[1][c.place(b, p)] = c.kc[1][c.place(b, p)]
            want_v[1][c.place(b, p)] = c.v[b, t]
    assert torch.equal(c.kc, want_k) and torch.equal(c.vc, want_v)
    # the same rows by the two calls it stands for
    two = Rows(6, 2, D, c.kv_len, c.n_new, paged, seed=D + rot)
    s = i32(c.kv_len)
    dreams.kv_append(two.cache(dreams), dreams.rope(two.k, r, start=s), two.v.contiguous(), s, i32(c.n_new), layer=1)
    assert torch.equal(two.kc, c.kc) and torch.equal(two.vc, c.vc)
    # K and V alone; and Q in place
    three = Rows(6, 2, D, c.kv_len, c.n_new, paged, seed=D + rot)
    assert dreams.kv_append_rope(three.cache(dreams), three.k, three.v, r, s, i32(c.n_new), layer=1) is None
    assert torch.equal(three.kc, c.kc) and torch.equal(three.vc, c.vc)
    q = c.q.contiguous()
    keep = q.clone()
    dreams.kv_append_rope(kv, c.k, c.v, r, s, i32(c.n_new), q=q, q_out=q, layer=1)
    for b in range(c.B):
        assert torch.equal(q[b, :c.n_new[b]], qo[b, :c.n_new[b]]) and torch.equal(q[b, c.n_new[b]:], keep[b, c.n_new[b]:])


def test_append_many_rows(dreams):
    c = Rows(32, 8, 128, [100, 0], [1501, 777], True, seed=3)
    r = dreams.Rotary.make(96, scaling="yarn", factor=4.0)
    s, n = i32(c.kv_len), i32(c.n_new)
    qo = dreams.kv_append_rope(c.cache(dreams), c.k, c.v, r, s, n, q=c.q)
    q, k = dreams.rope(c.q, r, start=s), dreams.rope(c.k, r, start=s)
    for b in range(2):
        m = c.n_new[b]
        assert torch.equal(qo[b, :m], q[b, :m])
        slot = torch.arange(m, device="cuda") + c.kv_len[b]
        page = c.table[b].long()[slot // 64]
        assert torch.equal(c.kc[0][page, slot % 64], k[b, :m]) and torch.equal(c.vc[0][page, slot % 64], c.v[b, :m])


def test_append_positions(dreams):
    """Trees stand at their depth in the slots of their nodes; given positions on several axes."""
    rng = np.random.default_rng(5)
    c = Rows(4, 2, 64, [70, 5, 0], [40, 64, 1], True, T_max=64, seed=4)
    parent = [[-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, 64)] for _ in range(3)]
    depth = [[0] * 64 for _ in range(3)]
    for b in range(3):
        for i in range(1, 64):
            depth[b][i] = depth[b][parent[b][i]] + 1
    parent[0][41] = 99  # past the rows in use
    r = dreams.Rotary.make(64)
    s, n = i32(c.kv_len), i32(c.n_new)
    pos = i32([[c.kv_len[b] + d for d in depth[b]] for b in range(3)])
    qo = dreams.kv_append_rope(c.cache(dreams), c.k, c.v, r, s, n, q=c.q, parent=i32(parent))
    d = Rows(4, 2, 64, [70, 5, 0], [40, 64, 1], True, T_max=64, seed=4)
    qp = dreams.kv_append_rope(d.cache(dreams), d.k, d.v, r, s, n, q=d.q, positions=pos)
    want = dreams.rope(c.q, r, positions=pos)
    for b in range(3):
        assert torch.equal(qo[b, :c.n_new[b]], want[b, :c.n_new[b]]) and torch.equal(qp[b, :c.n_new[b]], want[b, :c.n_new[b]])
    assert torch.equal(c.kc, d.kc) and torch.equal(c.vc, d.vc)
    m = dreams.Rotary.make(64, axis=[i % 3 for i in range(32)])
    three = torch.randint(0, 9999, (3, 3, 64), dtype=torch.int32, device="cuda")
    qm = dreams.kv_append_rope(d.cache(dreams), d.k, d.v, m, s, n, q=d.q, positions=three)
    want = dreams.rope(c.q, m, positions=three)
    for b in range(3):
        assert torch.equal(qm[b, :c.n_new[b]], want[b, :c.n_new[b]])


def test_append_bad_data(dreams):
    """Flags, and that a bad sequence, or a slot without a page, changes nothing of its own and nothing else's."""
    r = dreams.Rotary.make(64)
    for kv_len, n_new, parent, want, skipped in (
            ([-1, 10], [4, 4], None, dreams.DATA_BAD_KV_LEN, True), ([0, 10], [-1, 4], None, dreams.DATA_BAD_KV_LEN, True),
            ([0, 10], [9, 4], None, dreams.DATA_BAD_KV_LEN, True), ([126, 10], [8, 4], None, dreams.DATA_BAD_KV_LEN, True),
            ([0, 10], [4, 4], [-1, 0, 2, 0, 0, 0, 0, 0], dreams.DATA_BAD_PARENT, True), ([0, 10], [4, 4], [0, 0, 1, 0, 0, 0, 0, 0], dreams.DATA_BAD_PARENT, True),
            ([62, 10], [4, 4], None, dreams.DATA_BAD_PAGE, False)):
        c = Rows(4, 2, 64, [62, 10], [8, 8], True, T_max=8, seed=6)
        if want == dreams.DATA_BAD_PAGE:
            c.table[0, 1] = 10 ** 6
        before = c.kc.clone(), c.vc.clone()
        par = None if parent is None else i32([parent, [-1, 0, 0, 0, 0, 0, 0, 0]])
        qo = torch.full((2, 8, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        st = i32([0])
        dreams.kv_append_rope(c.cache(dreams), c.k, c.v, r, i32(kv_len), i32(n_new), q=c.q, q_out=qo, parent=par, status=st)
        assert int(st) == want
        for t in range(4):
            assert torch.equal(c.vc[0][c.place(1, 10 + t)], c.v[1, t])
            before[0][0][c.place(1, 10 + t)], before[1][0][c.place(1, 10 + t)] = c.kc[0][c.place(1, 10 + t)], c.v[1, t]
        if skipped:
            assert (qo[0] == 7.0).all()
        else:  # slots 62 and 63 have a page, 64 and 65 none
            assert torch.equal(qo[0, :4], dreams.rope(c.q, r, start=i32(kv_len))[0, :4])
            for t in range(2):
                before[0][0][c.place(0, 62 + t)], before[1][0][c.place(0, 62 + t)] = c.kc[0][c.place(0, 62 + t)], c.v[0, t]
        assert torch.equal(c.kc, before[0]) and torch.equal(c.vc, before[1])


def test_streams_and_graphs(dreams):
    """Behind a busy stream of its own, and captured and replayed on new inputs."""
    r = dreams.Rotary.make(128)
    c = Rows(28, 4, 128, [100], [1], True, seed=8)
    kv, s, n = c.cache(dreams), i32(c.kv_len), i32(c.n_new)
    want = dreams.kv_append_rope(kv, c.k, c.v, r, s, n, q=c.q).clone()
    side = torch.cuda.Stream()
    x = c.q.contiguous() * 0
    with torch.cuda.stream(side):
        busy = torch.randn((4096, 4096), device="cuda")
        for _ in range(20):
            busy = busy @ busy
            busy = busy / busy.norm()
        x.copy_(c.q)
    got = dreams.kv_append_rope(kv, c.k, c.v, r, s, n, q=x, stream=side)
    y = dreams.rope(x, r, start=s, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(y, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dreams.kv_append_rope(kv, c.k, c.v, r, s, n, q=x, q_out=out)
        y = dreams.rope(x, r, start=s)
    for at in (100, 17, 90):
        s.fill_(at)
        x.normal_()
        graph.replay()
        assert torch.equal(out, dreams.rope(x, r, start=s)) and torch.equal(y, out)
        assert torch.equal(c.vc[0][c.place(0, at)], c.v[0, 0])
