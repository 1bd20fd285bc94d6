"""Single tokens stored heads first ([B, H, 1, D]), and one KV head stored so: the same
bits as with dense tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def noise(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def heads_first(x):
    """The same memory as a [B, H, T, D] tensor's transpose(1, 2): T or H is 1."""
    B, T, H, D = x.shape
    return torch.as_strided(x, x.shape, (H * T * D, D, T * D, 1))


@pytest.mark.parametrize("B,Hq,Hkv,D", [(1, 28, 4, 128), (3, 8, 2, 64), (5, 64, 1, 64), (2, 16, 16, 128)])
def test_single_token_queries(dreams, B, Hq, Hkv, D):
    kv = dreams.KVCache(noise(B, 256, Hkv, D, seed=1), noise(B, 256, Hkv, D, seed=2))
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    L = torch.arange(100, 100 + B, dtype=torch.int32, device="cuda")
    q = noise(B, 1, Hq, D, seed=3)
    t = heads_first(q)
    for call in (lambda x: dreams.window_attention(x, kv, one, L, 0.1, 50, 2, want_lse=True)[:2],
                 lambda x: dreams.attention(x, kv, one, L, 0.1, dreams.ATTN_CAUSAL, want_lse=True)[:2]):
        for a, b in zip(call(q), call(t)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("Hkv,T", [(4, 1), (1, 1), (1, 9)])
def test_rows_appended_heads_first(dreams, Hkv, T):
    B, D = 3, 64
    k, v = noise(B, T, Hkv, D, seed=4), noise(B, T, Hkv, D, seed=5)
    L, n = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 63, 5], [T, T, 0]))
    got = []
    for a, b in ((k, v), (heads_first(k), heads_first(v)), (k, heads_first(v))):
        kv = dreams.KVCache(noise(B, 128, Hkv, D, seed=6), noise(B, 128, Hkv, D, seed=7))
        dreams.kv_append(kv, a, b, L, n)
        got.append((kv.k, kv.v))
    for x, y in got[1:]:
        assert torch.equal(x, got[0][0]) and torch.equal(y, got[0][1])
    assert torch.equal(got[0][0][1, 63:63 + T], k[1])
