"""The bounded waits of the tcgen05 kernel over 8-bit pages, made to run out on
purpose without any fault (the test hook dreams_test_set_stall): it flags
DREAMS_DATA_TIMEOUT, leaves the rows that it did not finish untouched and frees its
tensor memory; the next normal call is bit-identical to one made before the stall."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SENTINEL = 0x7F7F  # a bf16 bit pattern that no output takes here (3.4e38)


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    yield d
    d.test_set_stall(0, -1)


# one block of 128 rows per KV head (its keys split over a cluster), and pairs of blocks
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 24, 8, 2), (3, 300, 8, 2)])
@pytest.mark.parametrize("stall_at", [0, 1])
def test_wait_runs_out_then_recovers(dreams, B, T, Hq, Hkv, D, stall_at):
    g = torch.Generator().manual_seed(5)
    P, L, L8 = 64, 3001, 2944
    T = T if T * Hq // Hkv > 64 else 65  # (fewer rows have no such waits)
    q = torch.randn((B, T, Hq, D), generator=g).to(torch.bfloat16).cuda()
    k, v = (torch.randn((B * P, 64, Hkv, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    table = torch.arange(B * P, dtype=torch.int32, device="cuda").view(B, P)
    kv = dreams.KVCache(k, v, table)
    c = torch.zeros((B * P, 64, Hkv, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    kv8 = dreams.KV8Cache(c, c.clone(), torch.zeros((B * P, Hkv, 2), dtype=torch.int16, device="cuda"), table.clone())
    i32 = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    assert dreams.kv_quantize(kv, kv8, i32(0), i32(L)).tolist() == [L8] * B

    def run():
        out = torch.full(q.shape, SENTINEL, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        lse = torch.full(q.shape[:3], -7.0, dtype=torch.float32, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        dreams.kv8_attention(q, kv8, kv, i32(T), i32(L), i32(L8), D ** -0.5, out=out, lse=lse, status=st)
        torch.cuda.synchronize()
        return out.view(torch.int16), lse, int(st.item())

    ref, ref_lse, st = run()
    assert st == 0 and not (ref == SENTINEL).any()
    try:
        dreams.test_set_stall(dreams.TEST_ATTENTION, stall_at, 20_000_000)
        out, lse, st = run()
    finally:
        dreams.test_set_stall(0, -1)
    assert st == dreams.DATA_TIMEOUT
    assert (out == SENTINEL).all() and (lse == -7.0).all()  # every row spans more tiles than a CTA was given
    out, lse, st = run()
    assert st == 0 and torch.equal(out, ref) and torch.equal(lse, ref_lse)
