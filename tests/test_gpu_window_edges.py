"""Windowed attention at the ends of its number range, against the fp64 oracle:
scores that outgrow the first keys' by tens of nats, and large V with them.

Tolerance: that of tests/test_gpu_window.py (the bound is relative to |O| and
A = sum_j a_j |V_j|, so it holds at any scale of V). Queries are all ones here and a
key's elements nearly equal, so a score of x nats grows by like steps. The tensor
cores add 16 products at a time to an f32 sum that they may truncate, 2^-23 x each
of D / 16 <= 8 times: at most 1.2e-4 for 120 nats, and as much less for lower ones.
That is an error of the log-sum-exp, inside 1e-4 + 1e-6 |lse|, and a relative error
of a weight, inside 2e-4 A."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from test_gpu_window import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def rising(c, nats, vscale=1.0, seed=0):
    """Scores that rise with the slot, from about 0 to `nats`."""
    g = torch.Generator().manual_seed(seed)
    lift = torch.arange(c.cap, dtype=torch.float64) * (nats / min(n + m for n, m in zip(c.kv_len, c.q_len) if m))
    c.q = torch.ones_like(c.q)
    c.k = (lift.view(1, 1, -1, 1, 1) / (c.scale * c.D) + 0.02 * torch.randn(c.k.shape, generator=g)).to(torch.bfloat16)
    c.v = (c.v.float() * vscale).to(torch.bfloat16)
    return c


# one sequence's blocks split over clusters, the same for a tree, one block to a CTA, pairs of blocks, and a few rows
LAYOUTS = {"clusters": dict(Hq=8, Hkv=2, kv_len=[700], q_len=[70]), "tree": dict(Hq=8, Hkv=2, kv_len=[700], q_len=[60], tree=True),
           "blocks": dict(Hq=32, Hkv=8, kv_len=[700 + i for i in range(10)], q_len=[32 - i for i in range(10)], tree=True),
           "pairs": dict(Hq=32, Hkv=8, kv_len=[700 + i for i in range(10)], q_len=[64 - i for i in range(10)]),
           "rows": dict(Hq=8, Hkv=2, kv_len=[700], q_len=[3])}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nats,log2v", [(20, 86), (50, 70), (50, 86), (50, 0), (120, 0), (120, 86)])
def test_large_values_under_rising_scores(dreams, layout, D, nats, log2v):
    """Finite V up to 2^87 in magnitude gives finite outputs, however far the sums outgrow the first keys' reference."""
    c = rising(Case(7 * nats + D, D=D, window=10 ** 6, sinks=0, **LAYOUTS[layout]), nats, 2.0 ** log2v / 5)  # normals stay below 5
    c.check(c.run(dreams), n=40)


class Queue:
    """On the same CTAs one after the other: a long request of two blocks, whose rows from `slow` on are all done again key
    by key (their scores rise by 80 nats), `rounds` - 1 short requests of one block, and one of two blocks again."""
    Hq, Hkv, D, T, scale = 32, 8, 64, 64, 0.125

    def __init__(self, rounds, first, slow):
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        assert sms % self.Hkv == 0
        self.B = B = sms // self.Hkv * rounds + 1  # the first and the last sequence's heads fall on the same CTAs
        g = torch.Generator().manual_seed(3)
        self.lens = lens = [first] + [3 + b % 30 for b in range(B - 2)] + [70]
        self.n = n = [self.T] + [1 + (b * 7) % 32 for b in range(B - 2)] + [self.T]
        P, at = -(-(first + self.T) // 64), 0
        self.table = torch.full((B, P), -1, dtype=torch.int32)
        for b in range(B):
            for e in range(-(-(lens[b] + n[b]) // 64)):
                self.table[b, e] = at
                at += 1
        k, v = (torch.randn((at, 64, self.Hkv, self.D), generator=g) for _ in range(2))
        q = torch.randn((B, self.T, self.Hq, self.D), generator=g)
        k[:P] = (torch.arange(P * 64) * (80.0 / first) / (self.scale * self.D)).view(P, 64, 1, 1) + 0.02 * k[:P]
        q[0, :slow] *= 0.1  # scores of about 1
        q[0, slow:] = 1.0
        self.q, self.k, self.v = (x.to(torch.bfloat16) for x in (q, k, v))
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.gpu = self.q.cuda(), self.k.cuda(), self.v.cuda(), self.table.cuda(), i32(n), i32(lens)

    def run(self, dreams):
        q, k, v, table, n, lens = self.gpu
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:3], 7.0, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        dreams.window_attention(q, dreams.KVCache(k, v, table), n, lens, self.scale, 10 ** 6, out=out, lse=lse, status=st)
        torch.cuda.synchronize()
        return out, lse, int(st.item())

    def check(self, out, lse):
        out, lse, B, n = out.double().cpu().numpy(), lse.double().cpu().numpy(), self.B, self.n
        for b in {0, 1, 2, 19, 20, B // 2, B - 20, B - 2, B - 1}:
            assert (out[b, n[b]:] == 7.0).all() and (lse[b, n[b]:] == 7.0).all()
            own = self.table[b, self.table[b] >= 0].long()
            K, V = (x[own].reshape(-1, self.Hkv, self.D).double().numpy() for x in (self.k, self.v))
            sel = [(t, h) for t in sorted({0, n[b] // 2, n[b] - 1}) for h in range(0, self.Hq, 5)]
            ref = S.window_rows(self.q[b].double().numpy(), lambda s, h: (K[s, h], V[s, h]), self.lens[b], self.scale, 10 ** 6, 0,
                                lambda h: h // 4, None, sel)
            for (t, h), (o, a, z) in zip(sel, ref):
                err, tol = np.abs(out[b, t, h] - o), 1.02 * 2.0 ** -8 * (np.abs(o) + a) + 2e-4 * a + 1e-6
                assert (err <= tol).all(), (b, t, h, float((err / tol).max()))
                assert abs(lse[b, t, h] - z) <= 1e-4 + 1e-6 * abs(z), (b, t, h)
        for b in range(B):  # no row was left out
            assert (lse[b, :n[b]] != 7.0).all()


def test_one_block_of_a_pair_far_behind(dreams):
    """The second block's warps fall behind by more items than the kernel keeps scan results of."""
    c = Queue(22, 2000, 32)
    out, lse, st = c.run(dreams)
    assert st == 0
    c.check(out, lse)


def test_rows_done_again_are_no_stall(dreams):
    """Warps that redo rows keep the CTA's other warps waiting for much longer than the limit of a wait."""
    c = Queue(2, 4000, 0)
    c.run(dreams)
    t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    t[0].record()
    ref, ref_lse, st = c.run(dreams)
    t[1].record()
    torch.cuda.synchronize()
    ms = t[0].elapsed_time(t[1])
    assert st == 0 and ms > 8  # (so the limit below is far above a wait for products or copies)
    c.check(ref, ref_lse)
    try:
        dreams.test_set_stall(dreams.TEST_ATTENTION, 1 << 30, int(ms * 1e6 / 8))  # no copy is withheld
        out, lse, st = c.run(dreams)
    finally:
        dreams.test_set_stall(0, -1)
    assert st == 0 and torch.equal(out, ref) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("Hq,Hkv,D", [(28, 4, 128), (8, 2, 64), (8, 1, 128), (3, 3, 64)])
@pytest.mark.parametrize("kv_len", [[0, 1, 2, 5], [40, 700, 3000, 63]])
@pytest.mark.parametrize("tree", [False, True])
def test_eight_rows_keep_sixteen_bits_of_the_probabilities(dreams, Hq, Hkv, D, kv_len, tree):
    """At most 8 rows per KV head: outputs closer than one bf16 a probability could give them.

    Tolerance: the probabilities are held to 2^-16 (two bf16, the second rounded), at most 2^-20 of one is added so that
    none of the two is zero, and the f32 parts cost 2e-4 at most, all relative to A = sum_j a_j |V_j|; the one rounding of the
    output is 2^-8 |O|. A single bf16 would cost up to 2^-8 A."""
    n = 8 // (Hq // Hkv) if tree else 1
    c = Case(77 + D, Hq, Hkv, D, kv_len, [n] * 4, 2500, 2, tree=tree, paged=D == 64)
    out, lse = (x.double().cpu().numpy() for x in c.run(dreams))
    K, V = (x[0].double().numpy() for x in (c.k, c.v))
    for b in range(4):
        sel = [(t, h) for t in range(n) for h in range(0, Hq, 3)]
        ref = S.window_rows(c.q[b].double().numpy(), lambda s, g: (K[b, s, g], V[b, s, g]), kv_len[b], c.scale, 2500, 2,
                            lambda h: h // (Hq // Hkv), c.parent[b] if tree else None, sel)
        for (t, h), (o, a, z) in zip(sel, ref):
            err, tol = np.abs(out[b, t, h] - o), 1.02 * 2.0 ** -8 * np.abs(o) + (2e-4 + 2.0 ** -16 + 2.0 ** -20) * a + 1e-6
            assert (err <= tol).all(), (b, t, h, float((err / tol).max()))


@pytest.mark.parametrize("T,L", [(1, 0), (1, 5), (3, 300), (4, 15)])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
def test_an_infinity_that_a_row_sees_is_its_output(dreams, T, L, bad):
    """An infinity in V of a seen slot makes that element infinite, of that sign, whatever the weight; the others stay."""
    c = Case(5, 8, 2, 128, [L], [T], 200, 1)
    c.v[0, 0, L, :, 7] = bad  # the first new slot: every query sees it
    out, lse = c.run(dreams)
    assert (out[0, :T, :, 7] == bad).all()
    rest = [i for i in range(128) if i != 7]
    assert torch.isfinite(out[0, :T, :, rest]).all() and torch.isfinite(lse[0, :T]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("stall_at", [0, 1, 30])
def test_a_pairs_wait_runs_out_then_recovers(dreams, D, stall_at):
    """Copies withheld (the test hook) in the layout of tests/test_gpu_window_timeout.py that its shapes do not reach: more
    blocks than SMs, so pairs of them. Two items for some CTAs, about 25 tiles each: rows of an item whose tiles all came
    are those of the normal call, the others are untouched."""
    g = torch.Generator().manual_seed(6)
    B, T, Hq, Hkv, L = 24, 64, 32, 8, 3001
    q = torch.randn((B, T, Hq, D), generator=g).to(torch.bfloat16).cuda()
    k, v = (torch.randn((B, L + T + 63, Hkv, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    kv = dreams.KVCache(k, v)
    n, lens = (torch.full((B,), x, dtype=torch.int32, device="cuda") for x in (T, L))

    def run():
        out = torch.full(q.shape, 0x7F7F, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        lse = torch.full(q.shape[:3], -7.0, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        dreams.window_attention(q, kv, n, lens, D ** -0.5, 3000, 4, out=out, lse=lse, status=st)
        torch.cuda.synchronize()
        return out.view(torch.int16), lse, int(st.item())

    ref, ref_lse, st = run()
    assert st == 0 and not (ref == 0x7F7F).any()
    try:
        dreams.test_set_stall(dreams.TEST_ATTENTION, stall_at, 20_000_000)
        out, lse, st = run()
    finally:
        dreams.test_set_stall(0, -1)
    assert st == dreams.DATA_TIMEOUT
    done = lse != -7.0
    assert torch.equal(out[done], ref[done]) and torch.equal(lse[done], ref_lse[done])
    assert (out[~done] == 0x7F7F).all()
    assert not done.any() if stall_at < 2 else done.any() and not done.all()
    out, lse, st = run()
    assert st == 0 and torch.equal(out, ref) and torch.equal(lse, ref_lse)
