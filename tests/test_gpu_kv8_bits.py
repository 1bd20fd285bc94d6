"""How many bits of the probabilities count with few rows over 8-bit pages: 11. The softmax is
decided by a few keys, and elements are looked at whose terms nearly cancel, so that the
rounding of the output hides nothing.

Bound: a probability rounded to f16 is off by at most 2^-11 of itself (its step is 2^-10), to
bf16 by 2^-8; outputs are rounded to bf16. With A8 and A16 = sum_j a_j |V_j| over the slots
in 8 bits and those in bf16, whose probabilities are two bf16 with at most 8 rows (2^-16) and
one above that, an element may be off by 1.02 (2^-8 |O| + 2^-11 A8 + w A16) + 2e-4 A + 1e-6,
the last two for f32 scores and sums, as in test_gpu_kv8.py. The oracle with probabilities of
bf16 breaks the bound, so the kernel with such would."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from test_gpu_kv8 import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def bf16(x):
    return torch.tensor(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("D,G,T", [(128, 4, 1), (128, 8, 1), (128, 4, 4), (128, 4, 8), (64, 4, 2), (64, 8, 2), (64, 4, 16)])
def test_bits_of_the_probabilities(dreams, D, G, T):
    B, Hkv, L, end = 4, 2, 200, 192
    c = Case(D + G + T, G * Hkv, Hkv, D, [L] * B, [T] * B, [end] * B, kscale=4.0)
    out = c.run(dreams)[0].double().cpu().numpy()
    wide = 2.0 ** -16 if G * T <= 8 else 2.0 ** -8
    worse = 0
    for b in range(B):
        K, V = (x[0, b] for x in c.vals)
        q = c.q[b].double().numpy()
        for t in range(T):
            see = np.array(S.visible(t, L, c.window, 0))
            for h in range(G * Hkv):
                k, v = K[see, h // G], V[see, h // G]
                x = c.scale * (k @ q[t, h])
                p = np.exp(x - x.max())
                z = p.sum()
                o, terms = (p / z) @ v, (p / z)[:, None] * np.abs(v)
                a8, a16 = terms[see < end].sum(0), terms[see >= end].sum(0)
                tol = 1.02 * (2.0 ** -8 * np.abs(o) + 2.0 ** -11 * a8 + wide * a16) + 2e-4 * (a8 + a16) + 1e-6
                err = np.abs(out[b, t, h] - o)
                assert (err <= tol).all(), (b, t, h, float((err / tol).max()))
                worse += int((np.abs((bf16(p) / z) @ v - o) > tol).sum())
    assert worse > 0
