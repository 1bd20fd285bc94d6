"""rope in autograd: the gradient against the fp64 oracle's transposed turn and against
differences, gradients that are one value spread over the tensor, views, a second
derivative, positions that changed in between, and a step replayed from a graph.

Tolerance, as for rope itself: a gradient element is a sum of two f32 products with cosines
and sines that are off by some 2^-22 (the angle's 24 bits up to pi, and sincospif), so by at
most 1e-6 of factor (|u| + |v|); in bf16 it is rounded once more, by 2^-8 of its value:
eight bits, so values of [1, 2) lie 2^-7 apart and the nearest is at most 2^-8 away."""
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


def check(got, g, phases, pos, layout, factor, transpose):
    """got, g: [T, H, D] of one sequence."""
    u = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    got, g = got.double().cpu().numpy(), g.double().cpu().numpy()
    for t in range(g.shape[0]):
        want = R.rotate(g[t], phases, pos[t], layout, factor, transpose)
        size = np.abs(g[t])
        mag = size.copy()
        for a, b in R.pairs(len(phases), layout):
            mag[..., a] = mag[..., b] = size[..., a] + size[..., b]
        assert (np.abs(got[t] - want) <= u * np.abs(want) + 1e-6 * abs(factor) * mag + 1e-30).all(), t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,D", [(64, 64), (24, 96), (6, 10)])
@pytest.mark.parametrize("transpose", [False, True])
def test_gradient_of_a_weighted_sum(dreams, dtype, layout, rot, D, transpose):
    g = torch.Generator().manual_seed(rot)
    x, w = (torch.randn((2, 5, 3, D), generator=g).to(dtype).cuda() for _ in range(2))
    x.requires_grad_()
    r = dreams.Rotary.make(rot, layout=layout, scaling="yarn", factor=4.0, device="cuda")
    pos = torch.randint(-50, 1 << 20, (2, 5), generator=g).to(torch.int32)
    (dreams.rope(x, r, positions=pos.cuda(), transpose=transpose) * w).sum().backward()
    ph = [int(p) % 2 ** 64 for p in r.phase.tolist()]
    for b in range(2):
        check(x.grad[b], w[b], ph, pos[b].tolist(), layout, r.factor, not transpose)


def test_against_differences(dreams):
    """The map is linear: a step of any size gives its derivative. f32 sums of 64 values of some units: 1e-4."""
    g = torch.Generator().manual_seed(1)
    x, w, d = (torch.randn((1, 4, 2, 8), generator=g).cuda() for _ in range(3))
    x.requires_grad_()
    r, start = dreams.Rotary.make(8, base=100.0, device="cuda"), i32([7])
    f = lambda y: (dreams.rope(y, r, start=start) * w).sum()  # noqa: E731
    grad, = torch.autograd.grad(f(x), x)
    with torch.no_grad():
        assert abs(float((f(x + d) - f(x - d)) / 2 - (grad * d).sum())) < 1e-4


def test_spread_gradients_views_and_second_derivatives(dreams):
    r, start = dreams.Rotary.make(64, device="cuda"), i32([3, 90])
    ph = [int(p) % 2 ** 64 for p in r.phase.tolist()]
    qkv = torch.randn((2, 5, 9, 64), device="cuda", requires_grad=True)
    dreams.rope(qkv[:, :, 2:6], r, start=start).sum().backward()  # (the gradient comes with strides of zero)
    assert (qkv.grad[:, :, :2] == 0).all() and (qkv.grad[:, :, 6:] == 0).all()
    for b in range(2):
        check(qkv.grad[b, :, 2:6], torch.ones(5, 4, 64), ph, [int(start[b]) + t for t in range(5)], "half", 1.0, True)
    x, v = (torch.randn((2, 5, 4, 64), device="cuda", requires_grad=True) for _ in range(2))
    g, = torch.autograd.grad(dreams.rope(x, r, start=start), x, v, create_graph=True)
    c = torch.randn_like(v)
    back, = torch.autograd.grad(g, v, c)  # the gradient's gradient with respect to what came in is the turn itself
    for b in range(2):
        check(back[b], c[b], ph, [int(start[b]) + t for t in range(5)], "half", 1.0, False)


def test_positions_that_changed_since_are_noticed(dreams):
    r = dreams.Rotary.make(64, device="cuda")
    for kw in (dict(start=i32([3])), dict(positions=i32([[1, 5]]))):
        x = torch.randn((1, 2, 4, 64), device="cuda", requires_grad=True)
        y = dreams.rope(x, r, **kw)
        next(iter(kw.values())).add_(1)
        with pytest.raises(RuntimeError):
            y.sum().backward()


def test_a_step_replayed_from_a_graph(dreams):
    r, start = dreams.Rotary.make(64, device="cuda"), i32([3, 90])
    x, w = torch.randn((2, 5, 4, 64), device="cuda", requires_grad=True), torch.randn((2, 5, 4, 64), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(dreams.rope(x, r, start=start), x, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(dreams.rope(x, r, start=start), x, w)
    w.normal_()
    graph.replay()
    want = dreams.rope(w, r, start=start, transpose=True)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
