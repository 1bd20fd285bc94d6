"""The example examples/quantized_serving.py, all its parts together on a GPU, against a
shadow of the cache on the CPU: a list of K and V rows per sequence and layer, turned,
put into 8 bits, moved and attended in fp64.

Tolerances. A turned row is within 5e-7 (|u| + |v|) factor of the oracle's and one
rounding to bf16 (2^-8 of the value; test_gpu_rope.py derives both); from then on the shadow goes by the
row that the cache holds, and what is moved or put into 8 bits matches bit for bit.
Attention: probabilities and outputs are rounded to bf16 (u = 2^-8 each), so an element may
be off by u (|O| + A) with A = sum_j a_j |V_j|; f32 scores and sums add about 1e-4 A."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import rotary_kv8 as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -8


def _example():
    spec = importlib.util.spec_from_file_location("quantized_serving", os.path.join(ROOT, "examples", "quantized_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Shadow:
    def __init__(self, samples, layers):
        self.rows = [[[] for _ in range(samples)] for _ in range(layers)]  # [layer][sequence]: (K, V) per slot
        self.compared = self.quantized = self.ended = 0

    def __call__(self, event, **w):
        getattr(self, event)(**w)

    def near(self, got, x, pos, rotary, layout):
        """A turned row [H, D] against the oracle's."""
        phases = [p % 2 ** 64 for p in rotary.phase.tolist()]
        want = R.rotate(x, phases, pos, layout, rotary.factor)
        tol = U * np.abs(want)
        for a, b in R.pairs(len(phases), layout):
            s = 5e-7 * rotary.factor * (np.abs(x[:, a]) + np.abs(x[:, b]))
            tol[:, a] += s
            tol[:, b] += s
        assert (np.abs(got - want) <= tol).all()

    def layer(self, layer, q, k, v, turned, out, kv_len, len8, n_new, parent, rotary, layout, scale, pool, pool8):
        q, k, v, turned, out = (x.double().cpu().numpy() for x in (q, k, v, turned, out))
        table, table8 = pool.kv.page_table.cpu().numpy(), pool8.kv.page_table.cpu().numpy()
        ck, cv = pool.kv.k[layer].double().cpu().numpy(), pool.kv.v[layer].double().cpu().numpy()
        k8, v8, exps = pool8.kv.k[layer].view(torch.uint8).cpu().numpy(), pool8.kv.v[layer].view(torch.uint8).cpu().numpy(), pool8.kv.exps[layer].cpu().numpy()
        par = None if parent is None else parent.cpu().numpy()
        for b, (L, n, L8) in enumerate(zip(kv_len.tolist(), n_new.tolist(), len8.tolist())):
            rows = self.rows[layer][b]
            assert len(rows) >= L and L8 % 64 == 0 and L - L8 < 64
            del rows[L:]
            chains = []
            for t in range(n):
                a, chain = t, []
                while a >= 0:
                    chain.append(a)
                    a = int(par[b, a]) if par is not None else a - 1
                chains.append(chain[::-1])
                pos = L + len(chain) - 1
                pg, at = table[b, (L + t) // 64], (L + t) % 64
                assert np.array_equal(cv[pg, at], v[b, t])
                if n < 100 or t % 37 == 0:
                    self.near(ck[pg, at], k[b, t], pos, rotary, layout)
                    self.near(turned[b, t], q[b, t], pos, rotary, layout)
                rows.append((ck[pg, at], cv[pg, at]))
            for s in range(L):  # either cache holds what the shadow holds
                e, at = s // 64, s % 64
                if s < L8:
                    z = table8[b, e]
                    assert table[b, e] == -1
                    have = (R.decode(k8[z, at], exps[z, :, None, 0]), R.decode(v8[z, at], exps[z, :, None, 1]))
                else:
                    have = ck[table[b, e], at], cv[table[b, e], at]
                assert np.array_equal(have[0], rows[s][0]) and np.array_equal(have[1], rows[s][1]), (layer, b, s, L8)
            for t in range(n) if n < 100 else (0, 1, n // 2, n - 1):
                sees = list(range(L)) + [L + a for a in chains[t]]
                K, V = np.stack([rows[s][0] for s in sees]), np.stack([rows[s][1] for s in sees])
                G = q.shape[2] // K.shape[1]
                for h in range(q.shape[2]):
                    x = scale * K[:, h // G] @ turned[b, t, h]
                    a = np.exp(x - x.max())
                    a /= a.sum()
                    ref, A = a @ V[:, h // G], a @ np.abs(V[:, h // G])
                    assert (np.abs(out[b, t, h] - ref) <= 1.02 * U * (np.abs(ref) + A) + 2e-4 * A + 1e-6).all(), (layer, b, t, h)
                self.compared += 1

    def quantize(self, kv_len, len8, new_len8, pool, pool8):
        for b, (L, a, z) in enumerate(zip(kv_len.tolist(), len8.tolist(), new_len8.tolist())):
            assert z == L // 64 * 64
            for rows in (layer[b] for layer in self.rows):
                for s in range(a, z, 64):
                    page = rows[s:s + 64]
                    kv = []
                    for x in (np.stack([r[0] for r in page]), np.stack([r[1] for r in page])):
                        codes, es = R.quantize_page(x)
                        kv.append(R.decode(codes, es[None, :, None]))
                    rows[s:s + 64] = list(zip(kv[0], kv[1]))
                    self.quantized += 1

    def fork(self, kv_len, len8):
        assert len(set(len8.tolist())) == 1
        for layer in self.rows:
            assert kv_len.tolist() == [len(layer[0])] * len(layer)
            for b in range(1, len(layer)):
                layer[b] = list(layer[0])

    def step(self, path, accept_len, kv_len, new_kv_len):
        for layer in self.rows:
            for b, L in enumerate(kv_len.tolist()):
                nodes = path[b].tolist()[:new_kv_len.tolist()[b] - L]
                layer[b] = layer[b][:L] + [layer[b][L + i] for i in nodes]

    def end(self, pool, pool8):
        for p in (pool, pool8):
            assert (p.kv.page_table == -1).all() and (p.refcount == 0).all()
        self.ended += 1


@pytest.mark.parametrize("kw", [dict(samples=3, steps=14, prompt=310), dict(samples=2, D=128, Hq=7, Hkv=1, prompt=200, T=2, steps=5, max_path=3, seed=1,
                                                                            layout="interleaved", scaling="none"),
                                dict(samples=2, D=128, Hq=12, Hkv=3, prompt=64, T=40, steps=6, max_path=20, seed=2)])
def test_quantized_serving(kw):
    m = _example()
    shadow = Shadow(kw["samples"], 2)
    r = m.serve(watch=shadow, **kw)
    assert r["status"] == 0
    assert shadow.ended == 1
    prompt = kw["prompt"]
    assert shadow.compared == 2 * ((4 if prompt >= 100 else prompt) + kw["samples"] * kw.get("T", 24) * kw["steps"])  # layers; prompt's rows, trees'
    assert shadow.quantized == 2 * (prompt // 64 + sum(n // 64 - prompt // 64 for n in r["kv_len"]))
    assert r["len8"] == [n // 64 * 64 for n in r["kv_len"]]
    assert r["pages_held"] <= r["pages"] and r["pages8_held"] <= r["pages8"]
