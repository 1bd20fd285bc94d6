"""Refusals of the windowed-serving entry points on the host, before any launch
(no GPU): each case breaks one rule."""
import ctypes

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from paper_2606_00535_gb300 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dreams._lib()


P = 0x1000  # placeholder, never dereferenced: every call below fails validation
INV, UNS, WS = dreams.ERR_INVALID_ARG, dreams.ERR_UNSUPPORTED, dreams.ERR_WORKSPACE
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation cases use placeholder pointers")


def cache(D=128, paged=True, **kw):
    a = dict(k=P, v=P, n_layers=2, layer_stride=1 << 20, Hkv=2, D=D, capacity=256, page_table=P if paged else None,
             page_size=64 if paged else 0, pages_per_seq=4 if paged else 0, num_pages=16 if paged else 0)
    a.update(kw)
    return dreams._KVCache(*a.values())


def pool(**kw):
    a = dict(page_table=P, refcount=P, B=3, pages_per_seq=4, num_pages=16)
    a.update(kw)
    return dreams._PagePool(*a.values())


@needs_no_gpu
def test_window_attention_refusals(lib):
    def call(q=P, sb=8 * 512, st=512, kv=None, layer=0, parent=None, ql=P, kl=P, B=2, T=8, Hq=4, scale=0.1, window=4, sinks=0, out=P,
             lse=None):
        kv = cache() if kv is None else kv
        return lib.dreams_window_attention(q, sb, st, ctypes.byref(kv), layer, parent, ql, kl, B, T, Hq, scale, window, sinks, out, lse,
                                           None, None)

    for kw in (dict(q=None), dict(out=None), dict(ql=None), dict(kl=None), dict(q=P + 2), dict(out=P + 8), dict(lse=P + 2), dict(layer=2),
               dict(layer=-1), dict(B=0), dict(T=0), dict(T=(1 << 20) + 1), dict(parent=P, T=65), dict(Hq=3), dict(Hq=0), dict(Hq=2 * 129),
               dict(window=0), dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(st=504), dict(st=516), dict(sb=504), dict(kv=cache(k=None)), dict(kv=cache(v=P + 8)), dict(kv=cache(layer_stride=-8)),
               dict(kv=cache(layer_stride=4)), dict(kv=cache(capacity=255)), dict(kv=cache(num_pages=0))):
        assert call(**kw) == INV, kw
    assert call(kv=cache(D=96), st=384, sb=8 * 384) == UNS
    assert call(kv=cache(page_size=32, pages_per_seq=8)) == UNS


@needs_no_gpu
def test_page_calls_refusals(lib):
    bad_pools = [pool(page_table=None), pool(refcount=None), pool(refcount=P + 1), pool(B=0), pool(B=65536), pool(pages_per_seq=0),
                 pool(num_pages=0), pool(pages_per_seq=1 << 26)]
    for p in bad_pools:
        r = ctypes.byref(p)
        assert lib.dreams_kv_reserve(r, P, P, P, 1 << 30, None, None) == INV
        assert lib.dreams_kv_release(r, P, P, None, None) == INV
        assert lib.dreams_kv_fork(ctypes.byref(cache()), r, P, P, P, P, 1 << 30, None, None) == INV
        assert lib.dreams_kv_reserve_workspace_size(r) == 0 and lib.dreams_kv_fork_workspace_size(r) == 0
    r = ctypes.byref(pool())
    assert lib.dreams_kv_reserve(r, None, P, P, 1 << 30, None, None) == INV
    assert lib.dreams_kv_reserve(r, P, P + 1, P, 1 << 30, None, None) == INV
    assert lib.dreams_kv_release(r, P, None, None, None) == INV
    need = lib.dreams_kv_reserve_workspace_size(r)
    assert need >= 4 * (3 + 16)
    for ws, n in ((None, need), (P, need - 1), (P + 4, need)):
        assert lib.dreams_kv_reserve(r, P, P, ws, n, None, None) == WS
    need = lib.dreams_kv_fork_workspace_size(r)
    for ws, n in ((None, need), (P, need - 1), (P + 4, need)):
        assert lib.dreams_kv_fork(ctypes.byref(cache()), r, P, P, P, ws, n, None, None) == WS
    # the cache is not the pool's
    for kv in (cache(paged=False), cache(page_table=2 * P), cache(pages_per_seq=5, capacity=320), cache(num_pages=17)):
        assert lib.dreams_kv_fork(ctypes.byref(kv), r, P, P, P, P, need, None, None) == INV
    for a in ((None, P, P), (P, None, P), (P, P, None)):
        assert lib.dreams_kv_fork(ctypes.byref(cache()), r, *a, P, need, None, None) == INV


@needs_no_gpu
def test_row_calls_refusals(lib):
    def append(kv=None, layer=0, k=P, v=P, sb=8 * 256, st=256, kl=P, n=P, B=2, T=8):
        return lib.dreams_kv_append(ctypes.byref(cache() if kv is None else kv), layer, k, v, sb, st, kl, n, B, T, None, None)

    for kw in (dict(layer=2), dict(layer=-1), dict(k=None), dict(v=P + 8), dict(st=248), dict(st=260), dict(sb=248), dict(kl=None), dict(n=None),
               dict(B=0), dict(T=0), dict(kv=cache(D=12)), dict(kv=cache(page_size=32))):
        assert append(**kw) == INV, kw

    def prune(kv=None, B=2, keep=P, v0=0, n_vis=10, r=5, kl=P, ref=None, new=2 * P):
        return lib.dreams_kv_prune(ctypes.byref(cache() if kv is None else kv), B, keep, v0, n_vis, r, kl, ref, new, None, None)

    for kw in (dict(B=0), dict(keep=None), dict(v0=-1), dict(n_vis=-1, r=-1), dict(r=-1), dict(r=11), dict(kl=None), dict(new=None), dict(new=P),
               dict(ref=P + 2), dict(kv=cache(Hkv=0))):
        assert prune(**kw) == INV, kw


def test_binding_checks_before_any_call():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    kv = dreams.KVCache(z(4, 64, 2, 64), z(4, 64, 2, 64), i(2, 2))
    flat = dreams.KVCache(z(2, 64, 2, 64), z(2, 64, 2, 64))
    q = z(2, 3, 4, 64)
    att = lambda q=q, kv=kv, ql=i(2), kl=i(2), **kw: dreams.window_attention(q, kv, ql, kl, 0.1, 8, **kw)  # noqa: E731
    for err, kw in ((TypeError, dict(q=z(2, 3, 4, 64, dt=torch.float16))), (ValueError, dict(q=z(2, 3, 4, 128)[..., ::2])), (ValueError, dict(ql=i(1))),
                    (TypeError, dict(kl=z(2))), (ValueError, dict(q=z(3, 3, 4, 64), ql=i(3), kl=i(3))), (ValueError, dict(q=z(2, 3, 4, 128))),
                    (ValueError, dict(parent=i(2, 4))), (ValueError, dict(out=z(2, 3, 4, 32))), (TypeError, dict(out=z(2, 3, 4, 64, dt=torch.float32))),
                    (ValueError, dict(lse=z(2, 3, 5, dt=torch.float32))), (ValueError, dict())):  # the last: tensors on the CPU
        with pytest.raises(err):
            att(**kw)
    with pytest.raises(ValueError):
        dreams.PagePool(flat, i(4))
    with pytest.raises(ValueError):
        dreams.PagePool.empty(flat)
    with pytest.raises(ValueError):
        dreams.PagePool(kv, i(5))
    pool = dreams.PagePool(kv, i(4))
    for f in (lambda: dreams.kv_reserve(pool, i(1), i(2)), lambda: dreams.kv_release(pool, i(2), i(1)), lambda: dreams.kv_fork(pool, i(1), i(2)),
              lambda: dreams.kv_fork(pool, i(2), i(2), new_kv_len=i(1)), lambda: dreams.kv_reserve(pool, i(2), i(2))):
        with pytest.raises(ValueError):
            f()
    n = z(2, 3, 2, 64)
    for f in (lambda: dreams.kv_append(kv, n, z(2, 3, 2, 32), i(2), i(2)), lambda: dreams.kv_append(kv, z(2, 3, 4, 64), z(2, 3, 4, 64), i(2), i(2)),
              lambda: dreams.kv_append(kv, n, z(2, 3, 4, 64)[:, :, :2], i(2), i(2)), lambda: dreams.kv_append(kv, n, n, i(1), i(2)),
              lambda: dreams.kv_prune(kv, i(2, 3, 1), 0, 4, i(2)), lambda: dreams.kv_prune(kv, i(3, 3), 0, 4, i(3)),
              lambda: dreams.kv_prune(flat, i(2, 3), 0, 4, i(2), refcount=i(4)), lambda: dreams.kv_prune(kv, i(2, 3), 0, 4, i(2), refcount=i(3))):
        with pytest.raises(ValueError):
            f()
