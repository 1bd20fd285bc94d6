"""What the operators between a layer's projections and its attention cost: rotary positions, rows appended to the paged
cache with the rotation applied on the way, full pages of the cache put into 8 bits, and attention over a cache whose
full pages are held in 8 bits. Each case is one pass as a serving (or, for the rotation's gradient, a training) program
makes it; the plain forms are elementary torch operations in 32 bits, with angles in 64."""
import math
import random

import torch

own = False

PAGE = 64
DEV = "cuda"
FAR = 1 << 20  # positions of a long context


# ------------------------------------------------------------------ cases
def _rotary(rot, layout="half", scaling="none", factor=1.0, base=10000.0, axes=1):
    """rot: dimensions of a head that are rotated; layout: pairs (i, i + rot / 2) or (2 i, 2 i + 1); scaling by `factor`
    of a context of 4096 positions; axes: position axes (three for visual tokens: time, row, column)."""
    return {"rot": rot, "layout": layout, "scaling": scaling, "factor": factor, "base": base, "axes": axes}


def _rope(name, B, T, H, D, dtype, far, transpose, fused, **rotary):
    """far: positions are given and spread up to a million; otherwise they count on from each sequence's start. fused: x
    is a view of a projection that holds H more heads."""
    return {"name": name, "op": "rope", "B": B, "T": T, "H": H, "D": D, "dtype": dtype, "far": far, "transpose": transpose, "fused": fused,
            **_rotary(**rotary)}


def _append(name, B, T, t_lo, Hq, Hkv, D, lo, hi, tree, paged, **rotary):
    """T rows per sequence at most, t_lo the fewest, behind lo..hi committed slots; Q, K and V are views of one projection."""
    return {"name": name, "op": "append", "B": B, "T": T, "t_lo": t_lo, "Hq": Hq, "Hkv": Hkv, "D": D, "lo": lo, "hi": hi, "tree": tree, "paged": paged,
            **_rotary(**rotary)}


def _quantize(name, B, Hkv, D, layers, lo, hi, new_lo, new_hi):
    """Sequences of lo..hi slots in 8 bits already, and new_lo..new_hi committed slots behind them."""
    return {"name": name, "op": "quantize", "B": B, "Hkv": Hkv, "D": D, "layers": layers, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi}


def _attn(name, B, T, t_lo, Hq, Hkv, D, lo, hi, lag, tree=False, window=0, sinks=0):
    """lo..hi committed slots, all but the last `lag` pages or fewer in 8 bits; window 0: every slot is seen."""
    return {"name": name, "op": "attn", "B": B, "T": T, "t_lo": t_lo, "Hq": Hq, "Hkv": Hkv, "D": D, "lo": lo, "hi": hi, "lag": lag, "tree": tree,
            "window": window, "sinks": sinks}


def listed():
    return [
        # the query heads of one chat's next token: only latency counts
        _rope("rotation, one token", 1, 1, 28, 128, "bf16", False, False, False, rot=128),
        # gradients of a draft's queries in training: 32 bits, part of the head, an odd length, neighbouring pairs
        _rope("rotation's gradient, 32 bits", 4, 701, 32, 64, "f32", False, True, False, rot=48, layout="interleaved"),
        # queries of a prompt of 2880 visual and 512 text tokens, positions on three axes, a context stretched by 8
        _rope("rotation, 3392 tokens", 1, 3392, 32, 128, "bf16", True, False, True, rot=128, scaling="yarn", factor=8.0, axes=3),
        # one token's rows of one layer of the 28/4-head target
        _append("append, one token", 1, 1, 1, 28, 4, 128, 2000, 2000, False, True, rot=128),
        # one layer's rows of the batched verification step: 16 trees of 32 to 64 nodes
        _append("append, 16 trees", 16, 64, 32, 32, 8, 128, 1500, 6000, True, True, rot=128, base=500000.0),
        # chunks of 16 prompts, odd lengths, part of the head rotated
        _append("append, 16 chunks", 16, 2048, 1001, 32, 8, 128, 1500, 6000, False, True, rot=96, scaling="ntk", factor=4.0),
        # behind a batch's decode step: the sequences whose last page has filled up, eight layers
        _quantize("quantize, a page each", 16, 8, 128, 8, 1500, 6000, 64, 64),
        # a prompt of 3392 tokens goes into 8 bits, 32 layers of 32 heads
        _quantize("quantize, 3392 tokens", 1, 32, 128, 32, 0, 0, 3392, 3392),
        # the next token of one chat
        _attn("8-bit decode, one sequence", 1, 1, 1, 28, 4, 128, 2000, 2000, 0),
        # a full decode batch with contexts up to 32K
        _attn("8-bit decode, batch of 64", 64, 1, 1, 32, 8, 128, 1500, 32768, 2),
        # the batched verification step: 16 sequences, trees of 32 to 64 nodes
        _attn("8-bit trees, batch of 16", 16, 64, 32, 32, 8, 128, 1500, 6000, 1, tree=True),
        # chunks of four prompts on top of what is cached, head dim 64, odd lengths
        _attn("8-bit chunks, D 64", 4, 999, 701, 32, 8, 64, 1501, 6000, 2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng, D):
    scaling = rng.choice(["none", "none", "linear", "ntk", "yarn"])
    return {"rot": rng.choice([D, D, D // 2, 2 * rng.randint(2, D // 2)]), "layout": rng.choice(["half", "interleaved"]), "scaling": scaling,
            "factor": 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 40.0]), "base": rng.choice([10000.0, 500000.0, 1000000.0]),
            "axes": rng.choice([1, 1, 3])}


def draw(rng):
    op = rng.choice(["rope", "append", "append", "quantize", "attn", "attn", "attn"])
    Hq, Hkv, D = rng.choice([(28, 4, 128), (32, 8, 128), (32, 32, 128), (40, 40, 128), (32, 8, 64), (4, 4, 64), (16, 1, 128)])
    if op == "rope":
        T = _log(rng, 1, 3000)
        B = rng.randint(1, max(1, min(32, 4000 // T)))
        c = _rope("", B, T, rng.choice([Hq, Hkv]), D, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.5,
                  **_draw_rotary(rng, D))
    elif op == "append":
        tree = rng.random() < 0.3
        T = rng.randint(2, 64) if tree else _log(rng, 1, 1500)
        B = rng.randint(1, max(1, min(32, 6000 // T)))
        lo = _log(rng, 1, 4000)
        c = _append("", B, T, rng.randint(1, T), Hq, Hkv, D, lo, _log(rng, lo, 6000), tree, rng.random() < 0.8, **_draw_rotary(rng, D))
    elif op == "quantize":
        B = _log(rng, 1, 32)
        new_hi = _log(rng, PAGE, 3000)  # (some sequences of a batch may not have a full page)
        c = _quantize("", B, Hkv if Hkv * D <= 2048 else 8, D, rng.randint(1, 8), 0, rng.choice([0, _log(rng, 1, 4000)]),
                      _log(rng, 1, new_hi) if B > 1 else new_hi, new_hi)
    else:
        kind = rng.choice(["decode", "tree", "chunk"])
        window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 100, 4096), rng.choice([0, 1, 4, 70]))])
        lo, lag = _log(rng, 1, 8000), rng.choice([0, 0, 1, 5])
        hi = _log(rng, lo, 16000)
        if kind == "decode":
            B = _log(rng, 1, 32)
            T = rng.choice([1, 1, 2, 4])
            c = _attn("", B, T, T, Hq, Hkv, D, lo, hi if B > 1 else lo, lag, window=window, sinks=sinks)
        elif kind == "tree":
            B, T = _log(rng, 1, 10), rng.randint(5, 64)
            hi = min(hi, 6000)
            c = _attn("", B, T, rng.randint(1, T), Hq, Hkv, D, min(lo, hi), hi if B > 1 else min(lo, hi), lag, tree=True, window=window, sinks=sinks)
        else:
            T = _log(rng, 65, 1500)
            B = rng.randint(1, max(1, min(3, 1500 // T)))
            lo, hi = min(lo, 3000), min(hi, 3000)
            c = _attn("", B, T, rng.randint(1, T), Hq, Hkv, D, lo, hi if B > 1 else lo, lag, window=window, sinks=sinks)
    c.pop("name")
    return c


def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly, both ends included (n = 1: hi)."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


# ------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _parents(rng, T, T_max):
    """A draft tree of T nodes, numbered level by level, about ten to a level."""
    p, prev, at = [-1], [0], 1
    while at < T:
        n = min(T - at, rng.randint(6, 12))
        p += sorted(rng.choice(prev) for _ in range(n))
        prev = list(range(at, at + n))
        at += n
    return p + [-1] * (T_max - T)


def _table(need, g, pages=0):
    """Page table [B, P] with a page of its own, in random order, where `need`; -1 elsewhere. And how many pages there are, at
    least `pages`."""
    n = int(need.sum())
    pages = max(1, n, pages)
    table = torch.full(need.shape, -1, dtype=torch.int32, device=DEV)
    table[need] = torch.randperm(pages, generator=g, device=DEV)[:n].to(torch.int32)
    return table, pages


def _freq(c):
    """Radians a position turns each pair by, in 64 bits."""
    rot, base, s = c["rot"], c["base"], c["factor"]
    if c["scaling"] == "ntk":  # the base stretched so that the slowest pair turns s times slower
        base = base * s ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if c["scaling"] == "linear":
        f = [x / s for x in f]
    if c["scaling"] == "yarn":  # slow pairs interpolated, fast ones kept: by their turns over the original 4096 positions
        keep = [min(1.0, max(0.0, (4096 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
        f = [x * (k + (1 - k) / s) for x, k in zip(f, keep)]
    return f


def _gain(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "yarn" else 1.0


def _axis(c):
    """The position axis of each pair: a quarter of them time, the rest rows and columns."""
    n = c["rot"] // 2
    return [0 if i < n // 4 else 1 if i < n // 4 + (n - n // 4) // 2 else 2 for i in range(n)] if c["axes"] == 3 else [0] * n


def _put_rotary(s, c):
    s["freq"] = torch.tensor(_freq(c), dtype=torch.float64, device=DEV)
    s["axis"] = torch.tensor(_axis(c), dtype=torch.int64, device=DEV)
    s["gain"] = _gain(c)
    if own:
        import paper_2606_00535_gb300 as dreams
        s["rotary"] = dreams.Rotary.make(c["rot"], base=c["base"], layout=c["layout"], scaling=c["scaling"], factor=c["factor"], original=4096,
                                         axis=_axis(c) if c["axes"] == 3 else None, device=DEV)


def _to_pages(x, pages):
    """Rows [pages, 64, heads, D] as 8-bit codes and the power of two of each page and head: the smallest by which the
    largest value fits into +-448."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax((1, 3)))
    e = torch.where(m == 0, -110, e.int() - torch.where(m <= 0.875, 9, 8)).clamp(-110, 119)
    return (x * torch.exp2(-e.float())[:, None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn), e.to(torch.int16)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    s = dict(c)
    B = c["B"]
    if c["op"] == "rope":
        T, H, D = c["T"], c["H"], c["D"]
        x = _randn(g, B, T, 2 if c["fused"] else 1, H, D, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        s["x"] = x[:, :, 0]
        s["start"] = None if c["far"] else torch.randint(0, 30000, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["positions"] = None
        if c["far"]:
            p = torch.randint(0, FAR, (B, 1), generator=g, device=DEV) + torch.arange(T, device=DEV)
            s["positions"] = (p if c["axes"] == 1 else torch.stack([p, p + p % 40, p + p % 61])).to(torch.int32)
        elif c["axes"] == 3:
            p = s["start"].long()[:, None] + torch.arange(T, device=DEV)
            s["start"], s["positions"] = None, torch.stack([p, p + p % 40, p + p % 61]).to(torch.int32)
        _put_rotary(s, c)
        return s
    if c["op"] == "append":
        T, Hq, Hkv, D = c["T"], c["Hq"], c["Hkv"], c["D"]
        lens, n_new = _spread(c["lo"], c["hi"], B), _spread(c["t_lo"], T, B)
        rng.shuffle(lens)
        s["kv_len"], s["n_new"] = _ints(lens), _ints(n_new)
        P = -(-(c["hi"] + T) // PAGE)
        if c["paged"]:
            e = torch.arange(P, device=DEV) * PAGE
            s["table"], pages = _table(e < (s["kv_len"] + s["n_new"])[:, None], g, sum((x + T) // PAGE + 1 for x in lens))
            shape = (pages, PAGE, Hkv, D)
        else:
            s["table"], shape = None, (B, P * PAGE, Hkv, D)
        s["k"], s["v"] = _randn(g, *shape), _randn(g, *shape)
        qkv = _randn(g, B, T, Hq + 2 * Hkv, D)  # one projection
        s["q"], s["k_new"], s["v_new"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        s["q_out"] = torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device=DEV)
        s["parent"] = _ints([_parents(rng, t, T) for t in n_new]) if c["tree"] else None
        s["positions"] = None
        if c["axes"] == 3 and not c["tree"]:
            p = s["kv_len"].long()[:, None] + torch.arange(T, device=DEV)
            s["positions"] = torch.stack([p // 3, p // 3 + p % 40, p // 3 + p % 61]).to(torch.int32)
        _put_rotary(s, c if s["positions"] is not None else {**c, "axes": 1})
        if own:
            import paper_2606_00535_gb300 as dreams
            s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
        return s
    Hkv, D = c["Hkv"], c["D"]
    if c["op"] == "quantize":
        old = [x // PAGE * PAGE for x in _spread(c["lo"], c["hi"], B)]
        new = _spread(c["new_lo"], c["new_hi"], B)
        rng.shuffle(old)
        s["begin"], s["end"] = _ints(old), _ints([a + b for a, b in zip(old, new)])
        P = -(-(max(old) + max(new)) // PAGE)
        e = torch.arange(P, device=DEV) * PAGE
        a, b = s["begin"][:, None], s["end"][:, None]
        s["table"], pages = _table((e >= a) & (e < b), g)
        s["table8"], pages8 = _table(e + PAGE <= b, g)
        shape, shape8 = (c["layers"], pages, PAGE, Hkv, D), (c["layers"], pages8, PAGE, Hkv, D)
        spread = torch.exp2(torch.randint(-2, 3, (Hkv, 1), generator=g, device=DEV).float()).to(torch.bfloat16)  # heads differ in size
        s["k"], s["v"] = _randn(g, *shape) * spread, _randn(g, *shape) * spread
        s["k8"], s["v8"] = (torch.zeros(shape8, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2))
        s["exps"] = torch.zeros((c["layers"], pages8, Hkv, 2), dtype=torch.int16, device=DEV)
    else:
        T, Hq = c["T"], c["Hq"]
        lens, q_len = _spread(c["lo"], c["hi"], B), _spread(c["t_lo"], T, B)
        rng.shuffle(lens)
        len8 = [max(0, x // PAGE - rng.randint(0, c["lag"])) * PAGE for x in lens]
        s["kv_len"], s["q_len"], s["len8"] = _ints(lens), _ints(q_len), _ints(len8)
        P = -(-(c["hi"] + T) // PAGE)
        e = torch.arange(P, device=DEV) * PAGE
        L, L8, n = s["kv_len"][:, None], s["len8"][:, None], s["q_len"][:, None]
        seen = (e < L + n) & ((e + PAGE > L - c["window"] + 1) | (e < c["sinks"]) | (c["window"] == 0))  # the rest has been given back
        s["table8"], pages8 = _table(seen & (e < L8), g)
        s["table"], pages = _table(seen & (e >= L8), g)
        spread = torch.exp2(torch.rand((Hkv, D), generator=g, device=DEV) * 2 - 1)  # channels differ in size
        s["k8"], ek = _to_pages(torch.randn((pages8, PAGE, Hkv, D), generator=g, device=DEV) * spread, pages8)
        s["v8"], ev = _to_pages(torch.randn((pages8, PAGE, Hkv, D), generator=g, device=DEV) * spread, pages8)
        s["exps"] = torch.stack([ek, ev], -1).contiguous()
        s["k"], s["v"] = _randn(g, pages, PAGE, Hkv, D), _randn(g, pages, PAGE, Hkv, D)
        s["q"] = _randn(g, B, T, Hq, D)
        s["parent"] = _ints([_parents(rng, t, T) for t in q_len]) if c["tree"] else None
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, T, Hq), dtype=torch.float32, device=DEV)
        s["scale"] = D ** -0.5
    if own:
        import paper_2606_00535_gb300 as dreams
        s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
        s["kv8"] = dreams.KV8Cache(s["k8"], s["v8"], s["exps"], s["table8"])
    return s


# ------------------------------------------------------------------ plain forms
def _turn(s, x, pos, transpose=False):
    """x [B, T, H, D] in 32 bits turned by pos [B, T], or [axes, B, T]."""
    rot, n = s["rot"], s["rot"] // 2
    p = pos.double()[..., None] if pos.dim() == 2 else pos.double()[s["axis"]].permute(1, 2, 0)
    a = p * s["freq"]
    cos, sin = (torch.cos(a) * s["gain"]).float()[:, :, None], (torch.sin(a) * s["gain"]).float()[:, :, None]
    if transpose:
        sin = -sin
    x = x.float()
    if s["layout"] == "half":
        u, v = x[..., :n], x[..., n:rot]
        y = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    else:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _depth_and_kin(parent):
    """Depth of each node [B, T], and whether node a is an ancestor of t or t itself [B, T, T]: a tree of T <= 64 nodes is
    closed after six squarings of its parent relation."""
    B, T = parent.shape
    kin = torch.eye(T, dtype=torch.float32, device=DEV).expand(B, T, T).clone()
    kin += torch.nn.functional.one_hot((parent.long() + 1), T + 1)[:, :, 1:].float()
    kin = (kin > 0).float()
    kin = (torch.matrix_power(kin, 64) > 0) if T > 1 else kin > 0
    return kin.sum(2) - 1, kin


def _rows(table, cap, at):
    """Row numbers of slots at [B, N] in a paged or contiguous cache."""
    if table is None:
        return torch.arange(at.shape[0], device=DEV)[:, None] * cap + at
    return torch.gather(table.long(), 1, at // PAGE).clamp(min=0) * PAGE + at % PAGE


def _plain_append(s):
    T, L = s["T"], s["kv_len"].long()[:, None]
    t = torch.arange(T, device=DEV)
    real = t < s["n_new"][:, None]
    pos = s["positions"] if s["positions"] is not None else L + (_depth_and_kin(s["parent"])[0] if s["tree"] else t)
    q, k = _turn(s, s["q"], pos), _turn(s, s["k_new"], pos)
    s["q_out"].copy_(torch.where(real[:, :, None, None], q, s["q_out"].float()))
    cap = None if s["paged"] else s["k"].shape[1]
    rows = _rows(s["table"], cap, torch.where(real, L + t, 0))[real]
    s["k"].view(-1, s["Hkv"], s["D"])[rows] = k[real].to(torch.bfloat16)
    s["v"].view(-1, s["Hkv"], s["D"])[rows] = s["v_new"][real]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_quantize(s):
    e = torch.arange(s["table"].shape[1], device=DEV) * PAGE
    full = (e >= s["begin"][:, None]) & (e + PAGE <= s["end"][:, None])
    src, dst = s["table"][full].long(), s["table8"][full].long()
    for x, x8, i in ((s["k"], s["k8"], 0), (s["v"], s["v8"], 1)):
        p = x[:, src].flatten(0, 1)
        codes, ex = _to_pages(p, p.shape[0])
        x8.view(torch.uint8)[:, dst] = codes.view(torch.uint8).view(s["layers"], -1, *x.shape[2:])
        s["exps"][:, dst, :, i] = ex.view(s["layers"], -1, s["Hkv"])
    return {"k": s["k8"], "v": s["v8"], "exps": s["exps"], "len8": s["end"] // PAGE * PAGE}


def _plain_attn(s):
    B, T, Hq, Hkv, D, W, S = (s[x] for x in ("B", "T", "Hq", "Hkv", "D", "window", "sinks"))
    cap = s["table"].shape[1] * PAGE
    W = W or 2 * cap
    L, n, L8 = s["kv_len"].long(), s["q_len"].long(), s["len8"].long()
    t = torch.arange(T, device=DEV)
    real = t < n[:, None]
    if s["tree"]:
        depth, kin = _depth_and_kin(s["parent"])
        depth = depth.long()
    else:
        depth, kin = t.expand(B, T), (t[:, None] >= t).expand(B, T, T)
    pos = L[:, None] + depth  # of the queries, and of the keys in the new slots
    # the slots that any row may see: the sinks, then the window of the first query up to the last new slot
    span = min(W - 1 + T, cap)
    base = (L - W + 1).clamp(min=min(S, cap))
    slots = torch.cat([torch.arange(min(S, cap), device=DEV).expand(B, -1), base[:, None] + torch.arange(span, device=DEV)], 1)
    valid = slots < (L + n)[:, None]
    old = slots < L[:, None]
    node = (slots - L[:, None]).clamp(0, T - 1)
    kpos = torch.where(old, slots, torch.gather(pos, 1, node))
    near = (pos[:, :, None] - kpos[:, None, :] < W) | (kpos < S)[:, None, :]
    mine = old[:, None, :] | torch.gather(kin, 2, node[:, None, :].expand(B, T, -1))
    see = near & mine & valid[:, None, :] & real[:, :, None]
    in8 = valid & (slots < L8[:, None])
    r8, r16 = _rows(s["table8"], cap, torch.where(in8, slots, 0)), _rows(s["table"], cap, torch.where(valid & ~in8, slots, 0))

    def rows(x8, x, i):  # [B, NK, Hkv, D]
        a = x8.view(torch.uint8).view(-1, Hkv, D)[r8].view(torch.float8_e4m3fn).float()
        a *= torch.exp2(s["exps"][r8 // PAGE, :, i].float())[..., None]
        return torch.where(in8[:, :, None, None], a, x.view(-1, Hkv, D)[r16].float()).masked_fill_(~valid[:, :, None, None], 0)

    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    x = (q @ rows(s["k8"], s["k"], 0).permute(0, 2, 3, 1)) * s["scale"]
    x = x.view(B, Hkv, T, Hq // Hkv, -1).masked_fill(~see[:, None, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = (p.view(B, Hkv, -1, p.shape[-1]) @ rows(s["v8"], s["v"], 1).permute(0, 2, 1, 3)).view(B, Hkv, T, Hq // Hkv, D) / z
    lse = (m + torch.log(z))[..., 0]
    o, lse = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D), lse.permute(0, 2, 1, 3).reshape(B, T, Hq)
    s["out"].copy_(torch.where(real[:, :, None, None], o, s["out"].float()))
    s["lse"].copy_(torch.where(real[:, :, None], lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    s = state
    if own:
        import paper_2606_00535_gb300 as dreams
        if s["op"] == "rope":
            return {"y": dreams.rope(s["x"], s["rotary"], positions=s["positions"], start=s["start"], transpose=s["transpose"])}
        if s["op"] == "append":
            q = dreams.kv_append_rope(s["kv"], s["k_new"], s["v_new"], s["rotary"], s["kv_len"], s["n_new"], q=s["q"], q_out=s["q_out"],
                                      positions=s["positions"], parent=s["parent"])
            return {"q": q, "k": s["k"], "v": s["v"]}
        if s["op"] == "quantize":
            len8 = dreams.kv_quantize(s["kv"], s["kv8"], s["begin"], s["end"])
            return {"k": s["k8"], "v": s["v8"], "exps": s["exps"], "len8": len8}
        out, lse = dreams.kv8_attention(s["q"], s["kv8"], s["kv"], s["q_len"], s["kv_len"], s["len8"], s["scale"], window=s["window"] or None,
                                        sinks=s["sinks"], parent=s["parent"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    if s["op"] == "rope":
        pos = s["positions"] if s["positions"] is not None else s["start"].long()[:, None] + torch.arange(s["T"], device=DEV)
        return {"y": _turn(s, s["x"], pos, s["transpose"]).to(s["x"].dtype)}
    return _plain_append(s) if s["op"] == "append" else _plain_quantize(s) if s["op"] == "quantize" else _plain_attn(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, B, D = case, case["B"], case["D"]
    if c["op"] == "rope":
        n = B * c["T"] * c["H"]
        return {"bytes": 2 * n * D * (2 if c["dtype"] == "bf16" else 4), "flops": 3 * n * c["rot"]}
    if c["op"] == "append":
        rows = sum(_spread(c["t_lo"], c["T"], B))
        return {"bytes": rows * (c["Hq"] + 2 * c["Hkv"]) * D * 4, "flops": 3 * rows * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["op"] == "quantize":
        pages = sum(x // PAGE for x in _spread(c["new_lo"], c["new_hi"], B))
        values = 2 * pages * PAGE * c["layers"] * c["Hkv"] * D
        return {"bytes": max(4 * B, 3 * values + 4 * pages * c["layers"] * c["Hkv"]), "flops": 2 * values}
    W, S, head = c["window"] or 1 << 30, c["sinks"], c["Hkv"] * D
    lens, q_len = _spread(c["lo"], c["hi"], B), _spread(c["t_lo"], c["T"], B)
    small = wide = pairs = 0
    for L, n in zip(lens, q_len):  # which length goes with which query count is drawn: the sums hardly depend on it
        first, L8 = max(0, L - W + 1), max(0, L // PAGE * PAGE - c["lag"] * PAGE // 2)
        seen8 = max(0, L8 - first) + min(S, first, L8)
        small += seen8
        wide += L + n - first + min(S, first) - seen8
        for t in range(n):
            if c["tree"]:  # a node about t / 9 levels deep sees its few ancestors
                p, extra = L + t // 9, min(t // 9 + 1, W)
                lo = max(0, p - W + 1)
                pairs += max(0, L - lo) + min(S, lo, L) + extra
            else:
                lo = max(0, L + t - W + 1)
                pairs += L + t + 1 - lo + min(S, lo)
    rows = sum(q_len) * c["Hq"]
    return {"bytes": 2 * small * head + 4 * wide * head + rows * (D * 4 + 4), "flops": 4 * D * c["Hq"] * pairs}


# ------------------------------------------------------------------ 64 bits
def _turned(s, x, pos):
    """One sequence's rows x [T, H, D], in 64 bits, turned as complex numbers by pos [T] or [axes, T]."""
    rot, n = s["rot"], s["rot"] // 2
    p = pos.double().expand(3, -1)[s["axis"]].T if pos.dim() == 1 else pos.double()[s["axis"]].T
    w = torch.polar(torch.full((p.shape[0], n), s["gain"], dtype=torch.float64, device=DEV), p * s["freq"])[:, None]
    first, second = (slice(0, n), slice(n, rot)) if s["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y = x.double().clone()
    z = torch.complex(y[..., first].clone(), y[..., second].clone()) * (w.conj() if s.get("transpose") else w)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _levels(parent):
    d = []
    for q in parent:
        d.append(0 if q < 0 else d[q] + 1)
    return d


def _exact_attn(s):
    B, T, Hq, Hkv, D, W, S = (s[x] for x in ("B", "T", "Hq", "Hkv", "D", "window", "sinks"))
    W = W or 1 << 30
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((B, T, Hq), dtype=torch.float64, device=DEV)
    lens, counts, lens8 = s["kv_len"].tolist(), s["q_len"].tolist(), s["len8"].tolist()
    for b in range(B):
        L, n, L8 = lens[b], counts[b], lens8[b]
        par = s["parent"][b].tolist() if s["tree"] else list(range(-1, n - 1))
        depth = torch.tensor(_levels(par[:n]), device=DEV)
        kin = torch.zeros((n, n), dtype=torch.bool)
        for t in range(n):
            if s["tree"]:
                a = t
                while a >= 0:
                    kin[t, a] = True
                    a = par[a]
            else:
                kin[t, :t + 1] = True
        slot = torch.arange(L + n, device=DEV)
        slot = slot[(slot > L - W) | (slot < S)]
        at = torch.where(slot < L, slot, L + depth[(slot - L).clamp(min=0)])  # the keys' positions
        mask = torch.cat([torch.ones((n, int((slot < L).sum())), dtype=torch.bool, device=DEV), kin.to(DEV)], 1)
        mask &= ((L + depth)[:, None] - at < W) | (at < S)
        page8, page = s["table8"][b].long()[slot // PAGE], s["table"][b].long()[slot // PAGE]
        for g in range(Hkv):
            k, v = torch.empty((2, len(slot), D), dtype=torch.float64, device=DEV)
            for y, x8, x, i in ((k, s["k8"], s["k"], 0), (v, s["v8"], s["v"], 1)):
                a = slot < L8
                y[a] = x8.view(torch.uint8)[page8[a], slot[a] % PAGE, g].view(torch.float8_e4m3fn).double() * \
                    torch.exp2(s["exps"][page8[a], g, i].double())[:, None]
                y[~a] = x[page[~a], slot[~a] % PAGE, g].double()
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                w = (s["q"][b, :n, h].double() @ k.T) * s["scale"]
                w[~mask] = -math.inf
                lse[b, :n, h] = torch.logsumexp(w, 1)
                out[b, :n, h] = torch.softmax(w, 1) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    """From the definitions, sequence by sequence: rotations as products of complex numbers, codes as the values that they
    round, attention over the slots that each query sees."""
    s = prepare(case, seed)
    if case["op"] == "rope":
        pos = s["positions"] if s["positions"] is not None else s["start"][:, None] + torch.arange(s["T"], device=DEV)
        return {"y": torch.stack([_turned(s, s["x"][b], pos[..., b, :]) for b in range(s["B"])])}
    if case["op"] == "append":
        q, k, v = (s[x].double() for x in ("q_out", "k", "v"))
        for b, (L, n) in enumerate(zip(s["kv_len"].tolist(), s["n_new"].tolist())):
            if s["positions"] is not None:
                pos = s["positions"][:, b, :n]
            else:
                pos = L + torch.tensor(_levels(s["parent"][b].tolist()[:n]) if s["tree"] else list(range(n)), device=DEV)
            q[b, :n] = _turned(s, s["q"][b, :n], pos)
            slot = L + torch.arange(n, device=DEV)
            page, row = (s["table"][b].long()[slot // PAGE], slot % PAGE) if s["paged"] else (b, slot)
            k[page, row], v[page, row] = _turned(s, s["k_new"][b, :n], pos), s["v_new"][b, :n].double()
        return {"q": q, "k": k, "v": v}
    if case["op"] == "quantize":
        both = [s["k8"].double(), s["v8"].double()]
        for b, (lo, hi) in enumerate(zip(s["begin"].tolist(), s["end"].tolist())):
            for p in range(-(-lo // PAGE), hi // PAGE):
                a, z = int(s["table"][b, p]), int(s["table8"][b, p])
                for x, y in zip((s["k"], s["v"]), both):
                    w = x[:, a].double()
                    # (16-bit values: a ratio that is no power of two is at least 2^-9 of itself away from one)
                    e = torch.ceil(torch.log2(w.abs().amax((1, 3), keepdim=True) / 448.0) - 1e-6)
                    y[:, z] = w * torch.exp2(-e)
        return {"k": both[0], "v": both[1], "exps": None, "len8": None}
    return _exact_attn(s)
