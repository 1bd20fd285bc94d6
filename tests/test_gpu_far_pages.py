"""Pools whose last pages lie beyond 2^32 bytes and 2^32 values: rotated appends, pages into 8 bits
and attention over them give there, bit for bit, what they give in small pools."""
import pytest
import torch

pytestmark = pytest.mark.gpu
PAGES = 70_000  # of 64 slots, 8 heads of 128: 2^32 codes are 65,536 pages
HKV, D = 8, 128


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


@pytest.fixture(scope="module")
def far():
    """(k, v, k8, v8, exps): 28 GB, of which the tests touch a few pages."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory")
    shape = (PAGES, 64, HKV, D)
    k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k8, v8 = (torch.empty(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    yield k, v, k8, v8, torch.zeros((PAGES, HKV, 2), dtype=torch.int16, device="cuda")
    del k, v, k8, v8
    torch.cuda.empty_cache()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("T", [1, 12, 60])
def test_far_pages(dreams, far, T):
    """Pages from PAGES - 40 on against pages from 0 on."""
    g = torch.Generator(device="cuda").manual_seed(T)
    lens, P = [900, 1203], 21
    near = [torch.zeros((40, *x.shape[1:]), dtype=torch.uint8 if x.dtype == torch.float8_e4m3fn else x.dtype, device="cuda") for x in far]
    near[2], near[3] = near[2].view(torch.float8_e4m3fn), near[3].view(torch.float8_e4m3fn)
    fill = torch.randn((2, 40, 64, HKV, D), generator=g, device="cuda").to(torch.bfloat16)
    new = torch.randn((2, T, 32 + 2 * HKV, D), generator=g, device="cuda").to(torch.bfloat16)
    q, k_new, v_new = new.split([32, HKV, HKV], 2)
    ids = torch.randperm(40, generator=torch.Generator().manual_seed(T))
    results = []
    for pools, first in ((near, 0), (far, PAGES - 40)):
        k, v, k8, v8, exps = pools
        k[first:first + 40], v[first:first + 40] = fill
        table = (ids[:2 * P - 2].view(2, P - 1) + first).to(torch.int32).cuda()
        table8 = (ids.flip(0)[:2 * P - 2].view(2, P - 1) + first).to(torch.int32).cuda()
        kv, kv8 = dreams.KVCache(k, v, table), dreams.KV8Cache(k8, v8, exps, table8)
        rotary, kl, n, st = dreams.Rotary.make(D), i32(*lens), i32(T, T), i32(0)
        qr = dreams.kv_append_rope(kv, k_new, v_new, rotary, kl, n, q=q, status=st)
        len8 = dreams.kv_quantize(kv, kv8, i32(0, 64), i32(*lens), status=st)
        assert len8.tolist() == [896, 1152]
        dreams.kv_quantize(kv, kv8, i32(0, 0), i32(64, 64), status=st)
        out, lse = dreams.kv8_attention(qr, kv8, kv, n, kl, len8, D ** -0.5, want_lse=True, status=st)
        assert int(st) == 0 and torch.isfinite(out.float()).all()
        results.append((qr, out, lse, *(x[first:first + 40].clone().view(torch.uint8) for x in pools)))
    for i, (a, b) in enumerate(zip(*results)):
        if i >= 5:  # codes and powers: of the pages that were written
            written = torch.unique(ids.flip(0)[:2 * P - 2].view(2, P - 1)[:, :14]).cuda()
            a, b = a[written], b[written]
        assert torch.equal(a, b), i


def test_far_rows_of_a_tensor(dreams, far):
    """rope over rows 2^31 values and more apart, into a dense result and in place."""
    k = far[0].view(PAGES * 64, HKV * D)
    step = PAGES * 64 // 2 - 7
    x = k[::step][:2].view(2, 1, HKV, D)  # 2.3 billion values apart
    assert x.stride(0) > 2 ** 31
    x.copy_(torch.randn(x.shape, device="cuda"))
    rotary = dreams.Rotary.make(D)
    want = dreams.rope(x.contiguous(), rotary, start=i32(5, 70_000))
    assert torch.equal(dreams.rope(x, rotary, start=i32(5, 70_000)), want)
    dreams.rope(x, rotary, start=i32(5, 70_000), out=x)
    assert torch.equal(x, want)
