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


def test_one_block_of_a_pair_far_behind(dreams):
    """A long request of two blocks, whose second block's rows are all done again key by key, and behind it, on the same
    CTAs, over twenty requests of one block, then one of two blocks again: the second block's warps fall behind by
    more items than the kernel keeps scan results of."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    Hq, Hkv, D, T, scale = 32, 8, 64, 64, 0.125
    assert sms % Hkv == 0
    B = sms // Hkv * 22 + 1  # the first and the last sequence's heads fall on the same CTAs
    g = torch.Generator().manual_seed(3)
    lens, n = [2000] + [3 + b % 30 for b in range(B - 2)] + [70], [T] + [1 + (b * 7) % 32 for b in range(B - 2)] + [T]
    P = -(-(lens[0] + T) // 64)
    table, at = torch.full((B, P), -1, dtype=torch.int32), 0
    for b in range(B):
        for e in range(-(-(lens[b] + n[b]) // 64)):
            table[b, e] = at
            at += 1
    k, v = (torch.randn((at, 64, Hkv, D), generator=g) for _ in range(2))
    q = torch.randn((B, T, Hq, D), generator=g)
    # the first sequence: scores rise by 80 nats for the rows of its second block (sums above 2^100), by about 1 for the others
    lift = torch.arange(P * 64) * (80.0 / lens[0]) / (scale * D)
    k[:P] = lift.view(P, 64, 1, 1) + 0.02 * k[:P]
    q[0, :32] *= 0.1
    q[0, 32:] = 1.0
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    st = i32([0])
    dreams.window_attention(q.cuda(), dreams.KVCache(k.cuda(), v.cuda(), table.cuda()), i32(n), i32(lens), scale, 10 ** 6, out=out, lse=lse, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in [0, 1, 2, 19, 20, B // 2, B - 20, B - 2, B - 1]:
        assert (out[b, n[b]:] == 7.0).all() and (lse[b, n[b]:] == 7.0).all()
        K, V = (x[table[b, table[b] >= 0].long()].reshape(-1, Hkv, D).double().numpy() for x in (k, v))
        sel = [(t, h) for t in sorted({0, n[b] // 2, n[b] - 1}) for h in range(0, Hq, 5)]
        ref = S.window_rows(q[b].double().numpy(), lambda s, h: (K[s, h], V[s, h]), lens[b], scale, 10 ** 6, 0, lambda h: h // 4, None, sel)
        for (t, h), (o, a, z) in zip(sel, ref):
            err, tol = np.abs(out[b, t, h] - o), 1.02 * 2.0 ** -8 * (np.abs(o) + a) + 2e-4 * a + 1e-6
            assert (err <= tol).all(), (b, t, h, float((err / tol).max()))
            assert abs(lse[b, t, h] - z) <= 1e-4 + 1e-6 * abs(z), (b, t, h)
    for b in range(B):  # no row of the others was left out
        assert (lse[b, :n[b]] != 7.0).all()
