"""The example examples/windowed_serving.py, all its parts together on a GPU,
against a shadow of the cache on the CPU: a list of K and V rows per sequence
and layer, moved by list operations and attended in fp64.

Tolerance: as for the attention operator alone. Probabilities and outputs are
rounded to bf16 (u = 2^-8 each), so an element may be off by u (|O| + A) with
A = sum_j a_j |V_j|; f32 scores and sums add about 1e-4 A. Cache rows are moved,
never computed: they match bit for bit."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -8


def _example():
    spec = importlib.util.spec_from_file_location("windowed_serving", os.path.join(ROOT, "examples", "windowed_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Shadow:
    def __init__(self, samples, layers):
        self.rows = [[[] for _ in range(samples)] for _ in range(layers)]  # [layer][sequence]: (K, V) per slot
        self.compared = self.ended = 0

    def __call__(self, event, **w):
        getattr(self, event)(**w)

    def layer(self, layer, q, k, v, out, kv_len, n_new, parent, window, sinks, scale, pool):
        q, k, v, out = (x.double().cpu().numpy() for x in (q, k, v, out))
        table = pool.kv.page_table.cpu().numpy()
        ck, cv = pool.kv.k[layer].double().cpu().numpy(), pool.kv.v[layer].double().cpu().numpy()
        par = None if parent is None else parent.cpu().numpy()
        for b, (L, n) in enumerate(zip(kv_len.tolist(), n_new.tolist())):
            rows = self.rows[layer][b]
            assert len(rows) >= L
            del rows[L:]
            rows += [(k[b, t], v[b, t]) for t in range(n)]
            for t in range(n) if n < 100 else (0, 1, n // 2, n - 1):
                depth, anc = t, set(range(t + 1))
                if par is not None:
                    anc, x = {t}, t
                    while par[b, x] >= 0:
                        x = int(par[b, x])
                        anc.add(x)
                    depth = len(anc) - 1
                pos = L + depth
                sees = [s for s in range(L) if s < sinks or s > pos - window]
                if par is None:
                    sees += [L + a for a in sorted(anc) if L + a < sinks or a > t - window]
                else:
                    sees += [L + a for a in sorted(anc)]  # trees here are far less deep than the window
                for s in sees:  # the cache holds what the shadow holds, wherever a query looks
                    pg = table[b, s // 64]
                    assert pg >= 0
                    assert np.array_equal(ck[pg, s % 64], rows[s][0]) and np.array_equal(cv[pg, s % 64], rows[s][1])
                K, V = np.stack([rows[s][0] for s in sees]), np.stack([rows[s][1] for s in sees])
                G = q.shape[2] // K.shape[1]
                for h in range(q.shape[2]):
                    x = scale * K[:, h // G] @ q[b, t, h]
                    a = np.exp(x - x.max())
                    a /= a.sum()
                    ref, A = a @ V[:, h // G], a @ np.abs(V[:, h // G])
                    assert (np.abs(out[b, t, h] - ref) <= 1.02 * U * (np.abs(ref) + A) + 2e-4 * A + 1e-6).all(), (layer, b, t, h)
                self.compared += 1

    def prune(self, kept, v0, visual):
        keep = kept[0].tolist()
        for layer in self.rows:
            layer[0] = layer[0][:v0] + [layer[0][s] for s in keep] + layer[0][v0 + visual:]

    def fork(self, kv_len):
        for layer in self.rows:
            assert kv_len.tolist() == [len(layer[0])] * len(layer)
            for b in range(1, len(layer)):
                layer[b] = list(layer[0])

    def step(self, path, accept_len, kv_len, new_kv_len):
        for layer in self.rows:
            for b, L in enumerate(kv_len.tolist()):
                nodes = path[b].tolist()[:new_kv_len.tolist()[b] - L]
                layer[b] = layer[b][:L] + [layer[b][L + i] for i in nodes]

    def end(self, pool):
        assert (pool.kv.page_table == -1).all() and (pool.refcount == 0).all()
        self.ended += 1


@pytest.mark.parametrize("kw", [dict(samples=3, steps=3), dict(samples=2, D=128, Hq=7, Hkv=1, visual=130, keep=1, text=63, v0=0, window=77,
                                                              sinks=0, T=5, steps=4, max_path=5, seed=1)])
def test_windowed_serving(kw):
    m = _example()
    shadow = Shadow(kw["samples"], 2)
    r = m.serve(watch=shadow, **kw)
    assert r["status"] == 0
    assert shadow.ended == 1
    assert shadow.compared == 2 * (4 + kw["samples"] * kw.get("T", 24) * kw["steps"])  # layers; the prompt's rows, the trees'
    assert r["pages_held"] <= r["pages"]
