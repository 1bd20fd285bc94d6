"""Windowed attention at the ends of its number range, against the fp64 oracle:
scores that outgrow the first keys' by tens of nats, and large V with them.

Tolerance: that of tests/test_gpu_window.py (the bound is relative to |O| and
A = sum_j a_j |V_j|, so it holds at any scale of V). Queries are all ones here and a
key's elements nearly equal, so a score of x nats grows by like steps. The tensor
cores add 16 products at a time to an f32 sum that they may truncate, 2^-23 x each
of D / 16 <= 8 times: at most 1.2e-4 for 120 nats, and as much less for lower ones.
That is an error of the log-sum-exp, inside 1e-4 + 1e-6 |lse|, and a relative error
of a weight, inside 2e-4 A."""
import pytest
import torch

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
