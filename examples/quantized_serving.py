"""Speculative serving from a cache whose full pages are held in 8 bits, end to end on
synthetic data.

A prompt is prefilled, its full pages are put into 8 bits and their bf16 pages given
back, and the prompt is forked: several samples share its pages of either kind. Then
every sample runs verification steps with draft trees. Each layer's rows go into the
cache with the rotation of their positions applied on the way, attention reads the 8-bit
pages and the bf16 rows behind them, the accepted nodes' rows close up, and pages that
have filled up are put into 8 bits.

There is no model here: queries, keys, values and logits are seeded noise of a
model's shapes. `watch(event, **what)` is called after each part.

    python examples/quantized_serving.py
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


def serve(samples=4, layers=2, Hq=8, Hkv=2, D=64, prompt=500, T=24, steps=8, vocab=32, max_path=9, seed=0, layout="half", scaling="yarn",
          watch=None):
    """Runs one request; returns a summary."""
    dev = torch.device("cuda")
    rng = torch.Generator().manual_seed(seed)
    watch = watch or (lambda event, **what: None)

    def noise(*shape):
        return torch.randn(shape, generator=rng).to(torch.bfloat16).to(dev)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    P = -(-(prompt + steps * max_path + T) // PAGE) + 1
    # bf16 pages: the prompt's at first, later what is not full and the trees; 8-bit pages: the prompt's, shared, and the samples' own
    num_pages = P + samples * (-(-T // PAGE) + 2)
    num_pages8 = P + samples * (steps * max_path // PAGE + 2)
    shape, shape8 = (layers, num_pages, PAGE, Hkv, D), (layers, num_pages8, PAGE, Hkv, D)
    kv = dreams.KVCache(torch.zeros(shape, dtype=torch.bfloat16, device=dev), torch.zeros(shape, dtype=torch.bfloat16, device=dev),
                        torch.empty((samples, P), dtype=torch.int32, device=dev))
    kv8 = dreams.KV8Cache(torch.zeros(shape8, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn),
                          torch.zeros(shape8, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn),
                          torch.zeros((layers, num_pages8, Hkv, 2), dtype=torch.int16, device=dev),
                          torch.empty((samples, P), dtype=torch.int32, device=dev))
    pool, pool8 = dreams.PagePool.empty(kv), dreams.PagePool.empty(kv8)
    rotary = dreams.Rotary.make(D, base=10000.0, layout=layout, scaling=scaling, factor=4.0, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    scale = D ** -0.5
    zero, top = ints([0] * samples), ints([P * PAGE] * samples)

    def extend(kv_len, len8, n_new, T_max, parent=None):
        """Pages, rows and attention of n_new new tokens per sequence, layer by layer."""
        dreams.kv_reserve(pool, kv_len, n_new, status=status)
        for layer in range(layers):
            qkv = noise(samples, T_max, Hq + 2 * Hkv, D)  # a layer's fused projection
            q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
            turned = dreams.kv_append_rope(kv, k, v, rotary, kv_len, n_new, q=q, parent=parent, layer=layer, status=status)
            out, _ = dreams.kv8_attention(turned, kv8, kv, n_new, kv_len, len8, scale, parent=parent, layer=layer, status=status)
            watch("layer", layer=layer, q=q, k=k, v=v, turned=turned, out=out, kv_len=kv_len, len8=len8, n_new=n_new, parent=parent,
                  rotary=rotary, layout=layout, scale=scale, pool=pool, pool8=pool8)

    def quantize(kv_len, len8):
        """Pages that have filled up go into 8 bits, and their bf16 pages back."""
        dreams.kv_reserve(pool8, len8, kv_len // PAGE * PAGE - len8, status=status)
        new = dreams.kv_quantize(kv, kv8, len8, kv_len, status=status)
        watch("quantize", kv_len=kv_len, len8=len8, new_len8=new, pool=pool, pool8=pool8)
        dreams.kv_release(pool, zero, new, status=status)
        return new

    # the prompt, in the first row
    n_new = ints([prompt] + [0] * (samples - 1))
    extend(zero, zero, n_new, prompt)
    kv_len, len8 = n_new, quantize(n_new, zero)

    # a copy for every sample: of the table of 8-bit pages, and of the last, partly filled page
    first = ints([0] * samples)
    kv_len = dreams.kv_fork(pool, first, kv_len, status=status)
    len8 = dreams.kv_fork(pool8, first, len8, status=status)
    watch("fork", kv_len=kv_len, len8=len8)
    accepted = torch.zeros(samples, dtype=torch.int64, device=dev)
    for _ in range(steps):
        n_new = ints([T] * samples)
        parent = random_trees(rng, samples, T).to(dev)
        extend(kv_len, len8, n_new, T, parent)
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
        len8 = quantize(kv_len, len8)
    held, held8 = int((pool.refcount > 0).sum()), int((pool8.refcount > 0).sum())
    dreams.kv_release(pool, zero, top, status=status)
    dreams.kv_release(pool8, zero, top, status=status)
    watch("end", pool=pool, pool8=pool8)
    return {"status": int(status.item()), "kv_len": kv_len.tolist(), "len8": len8.tolist(), "accepted": accepted.tolist(), "steps": steps,
            "pages": num_pages, "pages_held": held, "pages8": num_pages8, "pages8_held": held8}


if __name__ == "__main__":
    r = serve()
    assert r["status"] == 0, f"device status {r['status']:#x}"
    print(f"{len(r['kv_len'])} samples, {r['steps']} steps: accepted {r['accepted']} draft tokens, lengths {r['kv_len']}, of which {r['len8']} "
          f"in 8 bits; {r['pages_held']} bf16 pages and {r['pages8_held']} of half their size held at the end")
