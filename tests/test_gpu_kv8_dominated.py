"""kv8_attention where a page weighs next to nothing beside others that the same warp has
read: a page marked as not finite still makes the rows that see it NaN (0 x NaN is a NaN),
and one whose V is that much larger still decides the result. And where dimensions of Q are
next to nothing beside others that no key has a part in. Enough lists that each is one CTA's, so that its warps walk over several tiles; 4, 16, 36
and 80 rows of a KV head, on both sides of every change of kernel."""
import numpy as np
import pytest
import torch

from oracle import rotary_kv8 as R
from oracle import serving as S
from test_gpu_kv8 import Case, U

pytestmark = pytest.mark.gpu
LONG, SHORT, END = 500, 1, 448  # slots of the four sequences looked at, and of the others; those in 8 bits


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def case(seed, D, T, **kw):
    return Case(seed, 32, 8, D, [LONG] * 4 + [SHORT] * 16, [T] * 4 + [1] * 16, [END] * 4 + [0] * 16, T_max=T, **kw)


def scale_page(c, j, b, e, up):
    """An 8-bit page of K (j = 0) or V (1) times 2^up, stored values and oracle's."""
    z = int(c.table8[b, e])
    c.exps[:, z, :, j] = torch.where(c.exps[:, z, :, j] == 32767, 32767, c.exps[:, z, :, j] + up)
    c.vals[j, :, b, 64 * e:64 * e + 64] *= 2.0 ** up


def scale_tail(c, j, up):
    """All of the bf16 slots."""
    x = c.k if j == 0 else c.v
    x *= 2.0 ** up
    for b in range(c.B):
        c.vals[j, :, b, c.len8[b]:] *= 2.0 ** up


@pytest.mark.parametrize("T", [1, 4, 9, 20])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("j", [0, 1])
def test_marked_pages_of_no_weight(dreams, T, D, j):
    """K of all pages but the marked one times 2^7: its keys score some hundred units below a row's largest, and their
    probabilities are zero in f32. Marked: a sequence's first page, one in the middle, its last."""
    mark = {(0, 0, j), (1, 3, j), (2, 6, j)}
    c = case(T + D, D, T, mark=mark)
    for b in range(4):
        for e in range(END // 64):
            if (b, e, j) not in mark:
                scale_page(c, 0, b, e, 7)
    scale_tail(c, 0, 7)
    out, lse = c.run(dreams)
    for b in range(3):
        assert torch.isnan(out[b]).all(), (b, int((~torch.isnan(out[b])).sum()))
    assert torch.isfinite(out[3:]).all() and torch.isfinite(lse[3:]).all()
    # f32 scores of D products of up to 4 units x 128, as in test_gpu_kv8.py's dominated softmax
    e = 2 * 8 * 128 * D * 2.0 ** -24
    sel = [(t, h) for t in range(T) for h in (0, 13, 31)]
    K, V = (x[0, 3] for x in c.vals)
    ref = S.window_rows(c.q[3].double().numpy(), lambda s, g: (K[s, g], V[s, g]), LONG, c.scale, c.window, 0, lambda h: h // 4, None, sel)
    for (t, h), (o, a, z) in zip(sel, ref):
        assert (np.abs(out[3, t, h].double().cpu().numpy() - o) <= 1.02 * U * (np.abs(o) + a) + (2e-4 + 2 * e) * a + 1e-6).all()


@pytest.mark.parametrize("T", [1, 4, 9, 20])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("weight", [10, 30, 45, 60, 90])
def test_pages_of_little_weight_and_large_values(dreams, T, D, weight):
    """Probabilities of some 2^-weight of the others' on pages whose V is 2^124 times theirs: first, in the middle, last, two
    of one sequence. The bound is that of test_gpu_kv8.py: it goes by the magnitudes that add up to the result."""
    c = case(T + D + weight, D, T, kscale=0.25)
    heavy = {(0, 0), (1, 3), (2, 6), (3, 1), (3, 4)}
    c.q[..., 0] = 8.0
    depth = weight / (8.0 * c.scale * 1.4427)  # dimension 0 of those pages' keys: scores lower by weight ln 2
    c.k[..., 0] = 0.0
    c.vals[0, ..., 0] = 0.0
    for b in range(4):
        for e in range(END // 64):
            z, at = int(c.table8[b, e]), slice(64 * e, 64 * e + 64)
            c.k8[0, z, :, :, 0] = 0
            if (b, e) in heavy:
                for h in range(8):
                    k = c.vals[0, 0, b, at, h]
                    k[:, 0] = -depth
                    code, es = R.quantize_page(k[:, None])
                    c.k8[0, z, :, h], c.exps[0, z, h, 0] = torch.tensor(code[:, 0]), int(es[0])
                    c.vals[0, 0, b, at, h] = R.decode(code[:, 0], es[0])
            scale_page(c, 1, b, e, 84 if (b, e) in heavy else -40)
    scale_tail(c, 1, -40)
    c.check(c.run(dreams), n=6)


@pytest.mark.parametrize("T", [1, 4, 9, 20])
@pytest.mark.parametrize("D", [64, 128])
def test_small_dimensions_of_q(dreams, T, D):
    """Eight dimensions of Q that are up to 2^30.6 times the others, where K is zero: the others' eight bits make the scores.
    (Whole down to 2^-24 of the largest alone, they would have two bits left, and the log-sum-exp be off by some thousandths.)"""
    c = case(T + D, D, T)
    c.q = torch.where(c.q < 0, -1.0, 1.0).to(c.q.dtype) * c.q.abs().clamp(min=0.5) * 2.0 ** -15
    c.q[..., :8] = torch.where(c.q[..., :8] < 0, -1.5, 1.5) * 2.0 ** 14
    c.k[..., :8] = 0.0
    c.k8[..., :8] = 0
    c.vals[0, ..., :8] = 0.0
    for b in range(4):
        for e in range(END // 64):
            scale_page(c, 0, b, e, 15)
    scale_tail(c, 0, 15)
    c.check(c.run(dreams), n=6)
