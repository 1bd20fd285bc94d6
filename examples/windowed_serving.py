"""Windowed speculative serving on a paged cache, end to end on synthetic data.

One request with an image is answered by several samples at once. Its prompt is
prefilled in one call per layer, the less important visual tokens are dropped
from the cache, and the prompt is forked: the samples share its pages. Then every
sample runs verification steps with draft trees: pages for the tree's nodes, their
K and V into every layer, sliding-window attention with sinks over cache and tree,
acceptance, and the pages that are no longer needed given back (what the step did
not use, and what has left the window).

There is no model here: queries, keys, values and logits are seeded noise of a
model's shapes. `watch(event, **what)` is called after each part.

    python examples/windowed_serving.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_00535_gb300 as dreams  # noqa: E402

PAGE = 64


def random_trees(rng, B, T):
    """parent [B, T]: every node hangs below one of the nine before it."""
    parent = torch.full((B, T), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(1, T):
            parent[b, i] = int(torch.randint(max(0, i - 9), i, (1,), generator=rng))
    return parent


def serve(samples=4, layers=2, Hq=8, Hkv=2, D=64, v0=7, visual=576, keep=288, text=90, T=24, steps=6, window=200, sinks=4,
          vocab=32, max_path=9, seed=0, watch=None):
    """Runs one request; returns a summary."""
    dev = torch.device("cuda")
    rng = torch.Generator().manual_seed(seed)
    watch = watch or (lambda event, **what: None)

    def noise(*shape):
        return torch.randn(shape, generator=rng).to(torch.bfloat16).to(dev)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    prompt = v0 + visual + text
    P = -(-(prompt + steps * max_path + T) // PAGE) + 1
    num_pages = P + samples * (-(-(max(window, T) + T) // PAGE) + 2)  # far fewer than samples * P
    kv = dreams.KVCache(torch.zeros((layers, num_pages, PAGE, Hkv, D), dtype=torch.bfloat16, device=dev),
                        torch.zeros((layers, num_pages, PAGE, Hkv, D), dtype=torch.bfloat16, device=dev),
                        torch.empty((samples, P), dtype=torch.int32, device=dev))
    pool = dreams.PagePool.empty(kv)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    scale = D ** -0.5
    begin = ints([sinks] * samples)
    top = ints([P * PAGE] * samples)

    def extend(kv_len, n_new, T_max, parent=None):
        """Pages, rows and attention of n_new new tokens per sequence, layer by layer."""
        dreams.kv_reserve(pool, kv_len, n_new, status=status)
        outs = []
        for layer in range(layers):
            qkv = noise(samples, T_max, Hq + 2 * Hkv, D)  # a layer's fused projection
            q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
            dreams.kv_append(kv, k, v, kv_len, n_new, layer=layer, status=status)
            out, _ = dreams.window_attention(q, kv, n_new, kv_len, scale, window, sinks, parent=parent, layer=layer, status=status)
            outs.append(out)
            watch("layer", layer=layer, q=q, k=k, v=v, out=out, kv_len=kv_len, n_new=n_new, parent=parent, window=window, sinks=sinks,
                  scale=scale, pool=pool)
        return outs

    # the prompt, in the first row
    zero = ints([0] * samples)
    n_new = ints([prompt] + [0] * (samples - 1))
    extend(zero, n_new, prompt)
    kv_len = n_new

    # its visual tokens that the draft's attention looks at most; the other rows are idle
    weights = torch.softmax(noise(1, Hq, 8, prompt).float(), -1)
    _, kept = dreams.visual_importance(weights, v0, visual, keep)
    shorter = dreams.kv_prune(kv, kept, v0, visual, kv_len, refcount=pool.refcount, status=status)
    watch("prune", kept=kept, v0=v0, visual=visual)
    kv_len = torch.cat([shorter, zero[1:]])
    dreams.kv_release(pool, kv_len, top, status=status)

    # a copy for every sample; then what the window has left behind goes
    kv_len = dreams.kv_fork(pool, ints([0] * samples), kv_len, status=status)
    watch("fork", kv_len=kv_len)
    accepted = torch.zeros(samples, dtype=torch.int64, device=dev)
    for _ in range(steps):
        dreams.kv_release(pool, begin, kv_len - window + 1, status=status)
        n_new = ints([T] * samples)
        parent = random_trees(rng, samples, T).to(dev)
        extend(kv_len, n_new, T, parent)
        tokens = torch.randint(0, vocab, (samples, T), generator=rng).to(torch.int32)
        logits = torch.randn((samples, T, vocab), generator=rng)
        for b in range(samples):  # a target that agrees with the draft more often than not
            for i in range(1, T):
                if float(torch.rand((), generator=rng)) < 0.5:
                    logits[b, int(parent[b, i]), int(tokens[b, i])] = 9.0
        tree = dreams.Tree(parent, tokens.to(dev), n_new, kv_len)
        step = dreams.verify_step(logits.to(dev), tree, kv, max_path, status=status)
        watch("step", path=step["path"], accept_len=step["accept_len"], kv_len=kv_len, new_kv_len=step["new_kv_len"])
        accepted += step["accept_len"]
        kv_len = step["new_kv_len"]
        dreams.kv_release(pool, kv_len, top, status=status)
    held = int((pool.refcount > 0).sum())
    dreams.kv_release(pool, zero, top, status=status)
    watch("end", pool=pool)
    return {"status": int(status.item()), "kv_len": kv_len.tolist(), "accepted": accepted.tolist(), "steps": steps, "pages": num_pages,
            "pages_held": held, "pages_unshared": samples * P}


if __name__ == "__main__":
    r = serve()
    assert r["status"] == 0, f"device status {r['status']:#x}"
    print(f"{len(r['kv_len'])} samples, {r['steps']} steps: accepted {r['accepted']} draft tokens, lengths {r['kv_len']}; "
          f"{r['pages_held']} pages held at the end of a pool of {r['pages']} ({r['pages_unshared']} without sharing and eviction)")
