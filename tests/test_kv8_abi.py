"""Refusals of rope, kv_append_rope, kv_quantize and kv8_attention on the host, before
any launch (no GPU): each case breaks one rule."""
import ctypes

import pytest
import torch

import paper_2606_00535_gb300 as dreams
from paper_2606_00535_gb300 import build as libbuild

P = 0x1000  # placeholder, never dereferenced: every call below fails validation
INV, UNS = dreams.ERR_INVALID_ARG, dreams.ERR_UNSUPPORTED
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation cases use placeholder pointers")


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dreams._lib()


def cache(D=128, paged=True, **kw):
    a = dict(k=P, v=P, n_layers=2, layer_stride=1 << 20, Hkv=2, D=D, capacity=256, page_table=P if paged else None,
             page_size=64 if paged else 0, pages_per_seq=4 if paged else 0, num_pages=16 if paged else 0)
    a.update(kw)
    return dreams._KVCache(*a.values())


def cache8(D=128, **kw):
    a = dict(k=P, v=P, exps=P, n_layers=2, layer_stride=1 << 20, Hkv=2, D=D, page_table=P, pages_per_seq=4, num_pages=16)
    a.update(kw)
    return dreams._KV8Cache(*a.values())


def rotary(**kw):
    a = dict(phase=P, axis=None, n_pairs=32, layout=0, factor=1.0)
    a.update(kw)
    return dreams._Rotary(*a.values())


BAD_ROTARY = [dict(phase=None), dict(phase=P + 4), dict(axis=P + 2), dict(n_pairs=0), dict(n_pairs=65), dict(layout=2), dict(layout=-1),
              dict(factor=float("nan")), dict(factor=float("inf"))]


@needs_no_gpu
def test_rope_refusals(lib):
    def call(x=P, xs=(4096, 512, 128), out=2 * P, ys=(4096, 512, 128), dtype=1, B=2, T=8, H=4, D=128, r=None, pos=None, axes=1, start=None):
        r = rotary() if r is None else r
        return lib.dreams_rope(x, *xs, out, *ys, dtype, B, T, H, D, ctypes.byref(r), pos,
                               axes, start, 0, None, None)

    for kw in [dict(x=None), dict(out=None), dict(dtype=2), dict(B=0), dict(B=65536), dict(T=0), dict(H=0), dict(D=0),
               dict(D=127), dict(D=514), dict(x=P + 1), dict(out=P + 1), dict(x=P + 2, dtype=0), dict(axes=0), dict(axes=5, pos=P), dict(axes=2),
               dict(pos=P, start=P), dict(pos=P + 2), dict(start=P + 1), dict(xs=(-1, 512, 128)), dict(xs=(1 << 38, 512, 128)), dict(ys=(4096, 512, 64)),
               dict(ys=(4096, 0, 128)), dict(ys=(2048, 512, 128)), dict(ys=(4096, 511, 128)), dict(out=P, xs=(8192, 512, 128)),
               dict(ys=(4096, 128, 128))] + [dict(r=rotary(**b)) for b in BAD_ROTARY]:
        assert call(**kw) == INV, kw


@needs_no_gpu
def test_append_rope_refusals(lib):
    def call(kv=None, layer=0, q=P, qs=(8 * 512, 512), qo=2 * P, Hq=4, k=P, ks=(8 * 256, 256), v=P, vs=(8 * 256, 256), r=None, pos=None, axes=1, par=None,
             kl=P, n=P, B=2, T=8):
        kv, r = cache() if kv is None else kv, rotary() if r is None else r
        return lib.dreams_kv_append_rope(ctypes.byref(kv), layer, q, *qs, qo, Hq, k, *ks, v, *vs, ctypes.byref(r), pos, axes, par, kl, n, B,
                                         T, None, None)

    for kw in [dict(layer=2), dict(layer=-1), dict(q=None), dict(qo=None), dict(Hq=0), dict(q=None, qo=None), dict(q=P + 8), dict(qo=P + 8),
               dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 8), dict(qs=(4096, 504)), dict(qs=(4096, 516)),
               dict(ks=(8 * 256, 248)), dict(vs=(248, 256)), dict(vs=(1 << 38, 256)), dict(q=P, qo=P, qs=(8192, 1024)), dict(pos=P, par=P),
               dict(axes=2), dict(axes=0), dict(axes=5, pos=P), dict(par=P, T=65, qs=(65 * 512, 512)), dict(par=P + 1), dict(pos=P + 2), dict(kl=None),
               dict(n=None), dict(kl=P + 2), dict(n=P + 1), dict(B=0), dict(B=65536), dict(T=0), dict(T=(1 << 20) + 1), dict(kv=cache(D=12)),
               dict(kv=cache(page_size=32)), dict(kv=cache(D=520))] + [dict(r=rotary(**b)) for b in BAD_ROTARY]:
        assert call(**kw) == INV, kw


@needs_no_gpu
def test_quantize_refusals(lib):
    def call(kv=None, kv8=None, B=2, begin=P, end=P, new=2 * P):
        kv, kv8 = cache() if kv is None else kv, cache8() if kv8 is None else kv8
        return lib.dreams_kv_quantize(ctypes.byref(kv), ctypes.byref(kv8), B, begin, end, new, None, None)

    for kw in [dict(B=0), dict(B=65536), dict(begin=None), dict(end=None), dict(new=None), dict(new=P), dict(begin=P + 2), dict(kv=cache(k=None)),
               dict(kv=cache(n_layers=3))] + [dict(kv8=cache8(**b)) for b in BAD_KV8]:
        assert call(**kw) == INV, kw
    assert call(kv=cache(D=96), kv8=cache8(D=96)) == UNS
    assert call(kv8=cache8(pages_per_seq=1 << 23)) == UNS


BAD_KV8 = [dict(k=None), dict(v=None), dict(exps=None), dict(k=P + 8), dict(v=P + 4), dict(exps=P + 2), dict(n_layers=0), dict(n_layers=1),
           dict(layer_stride=-16), dict(layer_stride=8), dict(Hkv=0), dict(Hkv=4), dict(D=64), dict(page_table=None), dict(page_table=P + 2),
           dict(pages_per_seq=0), dict(num_pages=0), dict(pages_per_seq=1 << 26)]


@needs_no_gpu
def test_attention_refusals(lib):
    def call(q=P, sb=8 * 512, st=512, kv8=None, kv=None, layer=0, parent=None, ql=P, kl=P, l8=P, B=2, T=8, Hq=4, scale=0.1, window=4, sinks=0, out=P,
             lse=None):
        kv, kv8 = cache() if kv is None else kv, cache8() if kv8 is None else kv8
        return lib.dreams_kv8_attention(q, sb, st, ctypes.byref(kv8), ctypes.byref(kv), layer, parent, ql, kl, l8, B, T, Hq, scale, window, sinks, out,
                                        lse, None, None)

    for kw in [dict(q=None), dict(out=None), dict(ql=None), dict(kl=None), dict(l8=None), dict(l8=P + 2), dict(q=P + 2), dict(lse=P + 2), dict(layer=2),
               dict(B=0), dict(T=0), dict(parent=P, T=65), dict(Hq=3), dict(window=0), dict(sinks=-1), dict(scale=0.0), dict(st=504),
               dict(kv=cache(k=None))] + [dict(kv8=cache8(**b)) for b in BAD_KV8]:
        assert call(**kw) == INV, kw
    assert call(kv=cache(D=96), kv8=cache8(D=96), st=384, sb=8 * 384) == UNS


def test_binding_checks_before_any_call():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c = lambda *s: torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    e = lambda *s: torch.zeros(s, dtype=torch.int16)  # noqa: E731
    kv = dreams.KVCache(z(4, 64, 2, 64), z(4, 64, 2, 64), i(2, 2))
    kv8 = dreams.KV8Cache(c(4, 64, 2, 64), c(4, 64, 2, 64), e(4, 2, 2), i(2, 2))
    dreams.PagePool(kv8, i(4))
    for f in (lambda: dreams.KV8Cache(c(4, 64, 2, 64), c(4, 64, 2, 32), e(4, 2, 2), i(2, 2)), lambda: dreams.KV8Cache(c(4, 32, 2, 64), c(4, 32, 2, 64), e(4, 2, 2), i(2, 2)),
              lambda: dreams.KV8Cache(c(4, 64, 2, 64), c(4, 64, 2, 64), e(4, 2), i(2, 2)), lambda: dreams.KV8Cache(c(4, 64, 2, 64), c(4, 64, 2, 64), e(4, 2, 2), i(4)),
              lambda: dreams.PagePool(kv8, i(5))):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        dreams.KV8Cache(z(4, 64, 2, 64), z(4, 64, 2, 64), e(4, 2, 2), i(2, 2))
    r = dreams.Rotary.make(64, device="cpu")
    x = z(2, 3, 4, 64)
    for err, f in ((TypeError, lambda: dreams.rope(x.half(), r)), (TypeError, lambda: dreams.rope(x[0], r)), (ValueError, lambda: dreams.rope(z(2, 3, 64, 4).transpose(2, 3), r)),
                   (ValueError, lambda: dreams.rope(x, r, positions=i(2, 4))), (ValueError, lambda: dreams.rope(x, r, positions=i(2, 3), start=i(2))),
                   (ValueError, lambda: dreams.rope(x, r, start=i(1))), (ValueError, lambda: dreams.rope(x, r, out=x.float())),
                   (ValueError, lambda: dreams.rope(x, r, out=z(2, 3, 64, 4).transpose(2, 3))), (ValueError, lambda: dreams.rope(x, r)),  # the last: on the CPU
                   (ValueError, lambda: dreams.Rotary(torch.zeros(3, dtype=torch.int64), axis=i(2))), (TypeError, lambda: dreams.Rotary(i(3))),
                   (ValueError, lambda: dreams.Rotary(torch.zeros(3, dtype=torch.int64), layout=3))):
        with pytest.raises(err):
            f()
    n = z(2, 3, 2, 64)
    ap = lambda k=n, v=n, kl=i(2), nn=i(2), **kw: dreams.kv_append_rope(kv, k, v, r, kl, nn, **kw)  # noqa: E731
    for err, kw in ((ValueError, dict(v=z(2, 3, 2, 32))), (ValueError, dict(k=x, v=x)), (ValueError, dict(kl=i(1))), (ValueError, dict(q_out=x)),
                    (ValueError, dict(q=z(2, 4, 4, 64))), (ValueError, dict(q=x, q_out=z(2, 3, 2, 64))), (TypeError, dict(q=x.float())),
                    (ValueError, dict(parent=i(2, 2))), (ValueError, dict(parent=i(2, 3), positions=i(2, 3))), (ValueError, dict(positions=i(3, 3))),
                    (ValueError, dict(k=z(2, 3, 2, 128), v=z(2, 3, 2, 128))), (ValueError, dict(k=z(3, 3, 2, 64), v=z(3, 3, 2, 64), kl=i(3), nn=i(3))),
                    (ValueError, dict(q=x))):  # the last: on the CPU
        with pytest.raises(err):
            ap(**kw)
    for f in (lambda: dreams.kv_quantize(kv, kv8, i(2), i(1)), lambda: dreams.kv_quantize(kv, kv8, i(3), i(3)), lambda: dreams.kv_quantize(kv, kv8, i(2), i(2), new_len8=i(1)),
              lambda: dreams.kv_quantize(kv, dreams.KV8Cache(c(4, 64, 1, 64), c(4, 64, 1, 64), e(4, 1, 2), i(2, 2)), i(2), i(2)), lambda: dreams.kv_quantize(kv, kv8, i(2), i(2))):
        with pytest.raises(ValueError):
            f()
    at = lambda q=x, ql=i(2), kl=i(2), l8=i(2), kv8=kv8, **kw: dreams.kv8_attention(q, kv8, kv, ql, kl, l8, 0.1, **kw)  # noqa: E731
    for err, kw in ((TypeError, dict(q=x.float())), (ValueError, dict(l8=i(1))), (TypeError, dict(l8=z(2))), (ValueError, dict(q=z(2, 3, 4, 128))),
                    (ValueError, dict(q=z(3, 3, 4, 64), ql=i(3), kl=i(3), l8=i(3))), (ValueError, dict(parent=i(2, 2))), (ValueError, dict(out=z(2, 3, 4, 32))),
                    (ValueError, dict(lse=z(2, 3, 5, dt=torch.float32))),
                    (ValueError, dict(kv8=dreams.KV8Cache(c(4, 64, 2, 64), c(4, 64, 2, 64), e(4, 2, 2), i(1, 2)))), (ValueError, dict())):
        with pytest.raises(err):
            at(**kw)
