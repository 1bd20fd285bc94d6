"""What the windowed-serving operators cost: sliding-window attention with sinks over the KV cache, and the page and row
movements of that cache (reserve, append, release, fork, prune). Each case is one pass as a serving program makes it; the
plain forms are elementary torch operations in 32 bits."""
import math
import random

import torch

own = False

PAGE = 64
DEV = "cuda"


# ------------------------------------------------------------------ cases
def _attn(name, B, T, Hq, Hkv, D, lo, hi, window, sinks, paged, tree=False, t_lo=None):
    """T: query tokens (or tree nodes) per sequence at most, t_lo the fewest; lo..hi: committed prefix lengths."""
    return {"name": name, "op": "attn", "B": B, "T": T, "t_lo": T if t_lo is None else t_lo, "Hq": Hq, "Hkv": Hkv, "D": D, "lo": lo, "hi": hi,
            "window": window, "sinks": sinks, "paged": paged, "tree": tree}


def _step(name, B, T, t_lo, Hkv, D, layers, lo, hi, window, sinks):
    return {"name": name, "op": "step", "B": B, "T": T, "t_lo": t_lo, "Hkv": Hkv, "D": D, "layers": layers, "lo": lo, "hi": hi, "window": window,
            "sinks": sinks}


def _fork(name, groups, width, Hkv, D, layers, lo, hi, best):
    """groups x width rows. best: every row of a group becomes its first row; else rows draw their parents within the group."""
    return {"name": name, "op": "fork", "groups": groups, "width": width, "Hkv": Hkv, "D": D, "layers": layers, "lo": lo, "hi": hi, "best": best}


def _prune(name, B, Hkv, D, layers, v0, n_vis, keep, text, paged):
    return {"name": name, "op": "prune", "B": B, "Hkv": Hkv, "D": D, "layers": layers, "v0": v0, "n_vis": n_vis, "keep": keep, "text": text,
            "paged": paged}


def listed():
    return [
        # the next token of one chat: the 28/4-head target after its 2000-token prompt; only latency counts
        _attn("decode, one sequence", 1, 1, 28, 4, 128, 2000, 2000, 1024, 4, False),
        # a full decode batch with prompts up to 32K, everything behind the window already evicted from the paged cache
        _attn("decode, batch of 64", 64, 1, 32, 8, 128, 1500, 32768, 4096, 4, True),
        # one draft tree against the 32-head target's prompt of 2880 visual and 512 text tokens
        _attn("tree, one sequence", 1, 60, 32, 32, 128, 3392, 3392, 1024, 4, False, tree=True),
        # the batched verification step: 16 sequences, trees of 32 to 64 nodes, paged cache
        _attn("tree, batch of 16", 16, 64, 32, 8, 128, 1500, 6000, 2048, 4, True, tree=True, t_lo=32),
        # prefill of the same prompt in one call
        _attn("prefill, 3392 tokens", 1, 3392, 32, 32, 128, 0, 0, 1024, 4, False),
        # chunks of four prompts on top of what is cached, head dim 64, odd lengths and an odd window
        _attn("prefill chunks, D 64", 4, 999, 32, 8, 64, 1501, 6000, 1999, 3, True, t_lo=701),
        # cache side of one verification step: pages for a 48-node tree, its rows into every layer, the unused tail returned
        _step("cache step, one tree", 1, 48, 48, 4, 128, 4, 2000, 2000, 1024, 4),
        # the same for 16 prompt chunks of up to 2048 tokens, eight layers
        _step("cache step, 16 chunks", 16, 2048, 1001, 8, 128, 8, 1500, 6000, 2048, 4),
        # best of 8: seven rows become copies of the prompt's row in a 32-layer, 32-head cache
        _fork("fork, 8 samples", 1, 8, 32, 128, 32, 3417, 3417, True),
        # beam reordering: 16 requests of 8 beams
        _fork("fork, 128 beams", 16, 8, 8, 128, 8, 1500, 6000, False),
        # the draft's one-layer cache keeps half of 1200 visual tokens
        _prune("prune, one layer", 1, 4, 128, 1, 17, 1200, 600, 800, True),
        # all 32 layers of the 32-head target keep half of 2880 visual tokens
        _prune("prune, 32 layers", 1, 32, 128, 32, 35, 2880, 1440, 512, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "step", "fork", "prune"])
    if op == "attn":
        Hq, Hkv, D = rng.choice([(28, 4, 128), (32, 8, 128), (32, 32, 128), (40, 40, 128), (32, 8, 64), (4, 4, 64), (16, 1, 128)])
        kind = rng.choice(["decode", "tree", "prefill"])
        window, sinks, paged = _log(rng, 100, 4096), rng.choice([0, 1, 4, 16, 70]), rng.random() < 0.5
        lo = _log(rng, 1, 8000)
        hi = _log(rng, lo, 16000)
        if kind == "decode":
            B = _log(rng, 1, 32)
            T = rng.choice([1, 1, 2, 4])
            c = _attn("", B, T, Hq, Hkv, D, lo, hi if B > 1 else lo, window, sinks, paged)
        elif kind == "tree":
            B = _log(rng, 1, 12)
            T = rng.randint(5, 64)
            c = _attn("", B, T, Hq, Hkv, D, lo, hi if B > 1 else lo, min(window, 2048), sinks, paged, tree=True, t_lo=rng.randint(1, T))
        else:
            T = _log(rng, 65, 2500)
            B = rng.randint(1, max(1, min(4, 2500 // T)))
            lo, hi = (0, 0) if rng.random() < 0.5 else (min(lo, 3000), min(max(hi, lo), 3000))
            c = _attn("", B, T, Hq, Hkv, D, lo, hi if B > 1 else lo, min(window, 1024), sinks, paged, t_lo=rng.randint(1, T))
    elif op == "step":
        T = _log(rng, 1, 1500)
        lo = _log(rng, 1, 3000)
        c = _step("", _log(rng, 1, 16), T, rng.randint(1, T), rng.choice([1, 4, 8]), rng.choice([64, 128]), rng.randint(1, 8), lo, _log(rng, lo, 6000),
                  _log(rng, 100, 4096), rng.choice([0, 4, 70]))
    elif op == "fork":
        lo = _log(rng, 1, 3000)
        c = _fork("", _log(rng, 1, 16), rng.randint(2, 8), rng.choice([1, 4, 8]), rng.choice([64, 128]), rng.randint(1, 8), lo, _log(rng, lo, 6000),
                  rng.random() < 0.5)
    else:
        n_vis = _log(rng, 2, 2880)
        c = _prune("", rng.randint(1, 4), rng.choice([1, 4, 8]), rng.choice([64, 128]), rng.randint(1, 8), rng.randint(0, 100), n_vis, rng.randint(1, n_vis),
                   _log(rng, 1, 2000), rng.random() < 0.5)
    c.pop("name")
    return c


def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly, both ends included (n = 1: hi)."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


# ------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype) if math.prod(shape) < 1 << 28 else \
        torch.empty(shape, device=DEV, dtype=dtype).normal_(generator=g)


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


def _depths(parent):
    d = []
    for q in parent:
        d.append(0 if q < 0 else d[q] + 1)
    return d


def _table(need, g):
    """Page table [B, P] with a page of its own, in random order, where `need`; -1 elsewhere. And how many pages there are."""
    n = int(need.sum())
    table = torch.full(need.shape, -1, dtype=torch.int32, device=DEV)
    table[need] = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    return table, n


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    s = dict(c)
    if c["op"] == "attn":
        B, T = c["B"], c["T"]
        lens = _spread(c["lo"], c["hi"], B)
        q_len = _spread(c["t_lo"], T, B)
        rng.shuffle(lens)
        s["kv_len"], s["q_len"] = _ints(lens), _ints(q_len)
        cap = -(-(c["hi"] + T) // PAGE) * PAGE
        s["q"] = _randn(g, B, T, c["Hq"], c["D"])
        if c["paged"]:
            e = torch.arange(cap // PAGE, device=DEV) * PAGE
            L, n = s["kv_len"][:, None].long(), s["q_len"][:, None].long()
            need = ((e + PAGE > L - c["window"] + 1) | (e < c["sinks"])) & (e < L + n)  # the rest has been evicted
            s["table"], pages = _table(need, g)
            shape = (pages, PAGE, c["Hkv"], c["D"])
        else:
            s["table"], shape = None, (B, cap, c["Hkv"], c["D"])
        s["k"], s["v"] = _randn(g, *shape), _randn(g, *shape)
        s["parent"] = _ints([_parents(rng, t, T) for t in q_len]) if c["tree"] else None
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, T, c["Hq"]), dtype=torch.float32, device=DEV)
        s["scale"] = c["D"] ** -0.5
        if own:
            import paper_2606_00535_gb300 as dreams
            s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
        return s
    if c["op"] == "step":
        B, T = c["B"], c["T"]
        lens, n_new = _spread(c["lo"], c["hi"], B), _spread(c["t_lo"], T, B)
        rng.shuffle(lens)
        s["kv_len"], s["n_new"] = _ints(lens), _ints(n_new)
        P = -(-(c["hi"] + T) // PAGE)
        e = torch.arange(P, device=DEV) * PAGE
        s["table"], used = _table(e < s["kv_len"][:, None], g)
        pages = used + B * (T // PAGE + 2)
        place = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        s["table"] = torch.where(s["table"] >= 0, place[s["table"].clamp(min=0).long()], s["table"])
        s["ref"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
        s["ref"][s["table"][s["table"] >= 0].long()] = 1
        shape = (c["layers"], pages, PAGE, c["Hkv"], c["D"])
        s["k"], s["v"] = _randn(g, *shape), _randn(g, *shape)
        # K and V of the new rows are views of each layer's fused projection
        s["new"] = [_randn(g, B, T, 2, c["Hkv"], c["D"]) for _ in range(c["layers"])]
        # what is left behind the window, and what the step did not need of the new slots (half of it was accepted)
        s["behind"] = (_ints([c["sinks"]] * B), _ints([max(0, x - c["window"] + 1) for x in lens]))
        s["unused"] = (_ints([x + t // 2 for x, t in zip(lens, n_new)]), _ints([P * PAGE] * B))
        if own:
            import paper_2606_00535_gb300 as dreams
            s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
            s["pool"] = dreams.PagePool(s["kv"], s["ref"])
        return s
    if c["op"] == "fork":
        G, N = c["groups"], c["width"]
        B = G * N
        per_group = _spread(c["lo"], c["hi"], G)
        rng.shuffle(per_group)
        s["kv_len"] = _ints([x for x in per_group for _ in range(N)])
        s["parent"] = _ints([gr * N + (0 if c["best"] else rng.randrange(N)) for gr in range(G) for _ in range(N)])
        P = max(per_group) // PAGE + 3
        e = torch.arange(P, device=DEV)
        full = (s["kv_len"].long() // PAGE)[:, None]
        first = (torch.arange(B, device=DEV) % N == 0)[:, None]
        if c["best"]:  # one row holds the prompt, the others are idle
            s["table"], used = _table((e <= full) & first, g)
        else:  # the beams of a request share the full pages and own their last one
            t, used = _table(((e < full) & first) | (e == full), g)
            lead = t.view(G, N, P)[:, :1].expand(G, N, P).reshape(B, P)
            s["table"] = torch.where(e < full, lead, t).contiguous()
        pages = used + B + 5
        s["ref"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
        s["ref"] += torch.bincount(s["table"][s["table"] >= 0].long(), minlength=pages).to(torch.int32)
        shape = (c["layers"], pages, PAGE, c["Hkv"], c["D"])
        s["k"], s["v"] = _randn(g, *shape), _randn(g, *shape)
        if own:
            import paper_2606_00535_gb300 as dreams
            s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
            s["pool"] = dreams.PagePool(s["kv"], s["ref"])
        return s
    B, n = c["B"], c["n_vis"]
    L = c["v0"] + n + c["text"]
    cap = -(-L // PAGE) * PAGE
    s["kv_len"] = _ints([L - i * (c["text"] // (2 * B)) for i in range(B)])
    pick = torch.stack([torch.randperm(n, generator=g, device=DEV)[: c["keep"]].sort().values for _ in range(B)])
    s["keep"] = (pick + c["v0"]).to(torch.int32).contiguous()
    if c["paged"]:
        need = torch.ones((B, cap // PAGE), dtype=torch.bool, device=DEV)
        s["table"], pages = _table(need, g)
        shape = (c["layers"], pages, PAGE, c["Hkv"], c["D"])
    else:
        s["table"], shape = None, (c["layers"], B, cap, c["Hkv"], c["D"])
    s["k"], s["v"] = _randn(g, *shape), _randn(g, *shape)
    if own:
        import paper_2606_00535_gb300 as dreams
        s["kv"] = dreams.KVCache(s["k"], s["v"], s["table"])
    return s


# ------------------------------------------------------------------ plain forms
def _depth_and_kin(parent):
    """Depth of each node [B, T], and whether node a is an ancestor of t or t itself [B, T, T]: a tree of T <= 64 nodes is
    closed after six squarings of its parent relation."""
    B, T = parent.shape
    kin = torch.eye(T, dtype=torch.float32, device=DEV).expand(B, T, T).clone()
    kin += torch.nn.functional.one_hot((parent.long() + 1), T + 1)[:, :, 1:].float()
    kin = (kin > 0).float()
    kin = (torch.matrix_power(kin, 64) > 0) if T > 1 else kin > 0
    return kin.sum(2) - 1, kin


def _plain_attn(s):
    B, T, Hq, Hkv, D, W, S = (s[x] for x in ("B", "T", "Hq", "Hkv", "D", "window", "sinks"))
    cap = s["table"].shape[1] * PAGE if s["paged"] else s["k"].shape[1]
    L, n = s["kv_len"].long(), s["q_len"].long()
    t = torch.arange(T, device=DEV)
    real = t < n[:, None]
    if s["tree"]:
        depth, kin = _depth_and_kin(s["parent"])
        depth, kin = depth.long(), kin
    else:
        depth, kin = t.expand(B, T), (t[:, None] >= t).expand(B, T, T)
    pos = L[:, None] + depth  # of the queries, and of the keys in the new slots
    # the slots that any row may see: the sinks, then the window of the first query up to the last new slot
    span = min(W - 1 + T, cap)
    base = (L - W + 1).clamp(min=S)
    slots = torch.cat([torch.arange(min(S, cap), device=DEV).expand(B, -1), base[:, None] + torch.arange(span, device=DEV)], 1)
    valid = (slots < (L + n)[:, None]) & ((slots >= base[:, None]) | (slots < S))
    old = slots < L[:, None]
    node = (slots - L[:, None]).clamp(0, T - 1)
    kpos = torch.where(old, slots, torch.gather(pos, 1, node))
    near = (pos[:, :, None] - kpos[:, None, :] < W) | (kpos < S)[:, None, :]
    mine = old[:, None, :] | torch.gather(kin, 2, node[:, None, :].expand(B, T, -1))
    see = near & mine & valid[:, None, :] & real[:, :, None]
    at = torch.where(valid, slots, 0)
    if s["paged"]:
        page = torch.gather(s["table"].long(), 1, at // PAGE).clamp(min=0)
        rows = page * PAGE + at % PAGE
    else:
        rows = torch.arange(B, device=DEV)[:, None] * cap + at
    k = s["k"].view(-1, Hkv, D)[rows].float().permute(0, 2, 3, 1)  # [B, Hkv, D, NK]
    v = s["v"].view(-1, Hkv, D)[rows].float().masked_fill(~valid[:, :, None, None], 0).permute(0, 2, 1, 3)
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    x = (q @ k) * s["scale"]
    x = x.view(B, Hkv, T, Hq // Hkv, -1).masked_fill(~see[:, None, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = (p.view(B, Hkv, -1, p.shape[-1]) @ v).view(B, Hkv, T, Hq // Hkv, D) / z
    lse = (m + torch.log(z))[..., 0]
    o, lse = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D), lse.permute(0, 2, 1, 3).reshape(B, T, Hq)
    s["out"].copy_(torch.where(real[:, :, None, None], o, s["out"].float()))
    s["lse"].copy_(torch.where(real[:, :, None], lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _reserve(s):
    table, ref = s["table"], s["ref"]
    e = torch.arange(table.shape[1], device=DEV)
    lo, hi = s["kv_len"].long()[:, None], (s["kv_len"] + s["n_new"]).long()[:, None]
    need = (table < 0) & (e >= lo // PAGE) & (e * PAGE < hi)
    free = torch.argsort((ref != 0).to(torch.int32), stable=True)  # the free pages first, in ascending order
    rank = (torch.cumsum(need.flatten().long(), 0) - 1).view_as(need).clamp(0, len(ref) - 1)
    table.copy_(torch.where(need, free[rank].to(torch.int32), table))
    ref.scatter_add_(0, free[rank].flatten(), need.flatten().to(torch.int32))


def _release(s, begin, end):
    table, ref = s["table"], s["ref"]
    e = torch.arange(table.shape[1], device=DEV) * PAGE
    drop = (table >= 0) & (e >= begin[:, None]) & (e + PAGE <= end[:, None])
    ref.scatter_add_(0, table.clamp(min=0).flatten().long(), -drop.flatten().to(torch.int32))
    table.masked_fill_(drop, -1)


def _append(s, layer):
    new, T = s["new"][layer], s["T"]
    t = torch.arange(T, device=DEV)
    at = s["kv_len"].long()[:, None] + t
    real = t < s["n_new"][:, None]
    page = torch.gather(s["table"].long(), 1, torch.where(real, at // PAGE, 0)).clamp(min=0)
    rows = (page * PAGE + at % PAGE)[real]
    s["k"][layer].view(-1, s["Hkv"], s["D"])[rows] = new[:, :, 0][real]
    s["v"][layer].view(-1, s["Hkv"], s["D"])[rows] = new[:, :, 1][real]


def _plain_step(s):
    _reserve(s)
    for layer in range(s["layers"]):
        _append(s, layer)
    _release(s, *s["behind"])
    _release(s, *s["unused"])


def _plain_fork(s):
    table, ref = s["table"], s["ref"]
    B, P = table.shape
    e = torch.arange(P, device=DEV)
    parent = s["parent"].long()
    rows = torch.arange(B, device=DEV)
    first = torch.full((B,), B, device=DEV).scatter_reduce_(0, parent, rows, "amin")
    keeps = (first[parent] == rows)[:, None]
    L = s["kv_len"].long()[parent]
    src = table[parent]
    full, tail = (L // PAGE)[:, None], (L % PAGE)[:, None]
    after = torch.where(keeps | (e < full), src, -1)
    ref.zero_()
    ref.scatter_add_(0, after.clamp(min=0).flatten().long(), (after >= 0).flatten().to(torch.int32))
    need = ~keeps & (e == full) & (tail > 0) & (src >= 0)
    free = torch.argsort((ref != 0).to(torch.int32), stable=True)
    rank = (torch.cumsum(need.flatten().long(), 0) - 1).view_as(need).clamp(0, len(ref) - 1)
    fresh = free[rank]
    ref.scatter_add_(0, fresh.flatten(), need.flatten().to(torch.int32))
    table.copy_(torch.where(need, fresh.to(torch.int32), after))
    slot = torch.arange(PAGE, device=DEV)
    move = (need[:, :, None] & (slot < tail[:, :, None]))
    a = (src.long()[:, :, None] * PAGE + slot)[move]
    b = (fresh[:, :, None] * PAGE + slot)[move]
    for x in (s["k"], s["v"]):
        y = x.view(s["layers"], -1, s["Hkv"], s["D"])
        y[:, b] = y[:, a]
    return s["kv_len"][parent]


def _plain_prune(s):
    B, r, n, v0 = s["B"], s["keep"].shape[1], s["n_vis"], s["v0"]
    L = s["kv_len"].long()
    most = (s["table"].shape[1] * PAGE if s["paged"] else s["k"].shape[2])
    rest = torch.arange(v0 + n, most, device=DEV).expand(B, -1)
    src = torch.cat([s["keep"].long(), rest], 1)
    dst = (v0 + torch.arange(src.shape[1], device=DEV)).expand(B, -1)
    live = src < L[:, None]
    if s["paged"]:
        at = lambda x: torch.gather(s["table"].long(), 1, x // PAGE) * PAGE + x % PAGE  # noqa: E731
    else:
        at = lambda x: torch.arange(B, device=DEV)[:, None] * most + x  # noqa: E731
    a, b = at(src)[live], at(dst)[live]
    for x in (s["k"], s["v"]):
        y = x.view(s["layers"], -1, s["Hkv"], s["D"])
        y[:, b] = y[:, a]
    return s["kv_len"] - (n - r)


def run(state):
    s = state
    if own:
        import paper_2606_00535_gb300 as dreams
        if s["op"] == "attn":
            out, lse = dreams.window_attention(s["q"], s["kv"], s["q_len"], s["kv_len"], s["scale"], s["window"], s["sinks"], parent=s["parent"],
                                               out=s["out"], lse=s["lse"])
            return {"out": out, "lse": lse}
        if s["op"] == "step":
            dreams.kv_reserve(s["pool"], s["kv_len"], s["n_new"])
            for layer in range(s["layers"]):
                new = s["new"][layer]
                dreams.kv_append(s["kv"], new[:, :, 0], new[:, :, 1], s["kv_len"], s["n_new"], layer=layer)
            dreams.kv_release(s["pool"], *s["behind"])
            dreams.kv_release(s["pool"], *s["unused"])
            return {"k": s["k"], "v": s["v"], "table": s["table"], "ref": s["ref"]}
        if s["op"] == "fork":
            new_len = dreams.kv_fork(s["pool"], s["parent"], s["kv_len"])
            return {"k": s["k"], "v": s["v"], "table": s["table"], "ref": s["ref"], "kv_len": new_len}
        new_len = dreams.kv_prune(s["kv"], s["keep"], s["v0"], s["n_vis"], s["kv_len"])
        return {"k": s["k"], "v": s["v"], "kv_len": new_len}
    if s["op"] == "attn":
        return _plain_attn(s)
    if s["op"] == "step":
        _plain_step(s)
        return {"k": s["k"], "v": s["v"], "table": s["table"], "ref": s["ref"]}
    new_len = _plain_fork(s) if s["op"] == "fork" else _plain_prune(s)
    if s["op"] == "fork":
        return {"k": s["k"], "v": s["v"], "table": s["table"], "ref": s["ref"], "kv_len": new_len}
    return {"k": s["k"], "v": s["v"], "kv_len": new_len}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "attn":
        B, W, S, row = c["B"], c["window"], c["sinks"], c["Hkv"] * c["D"] * 2
        lens, q_len = _spread(c["lo"], c["hi"], B), _spread(c["t_lo"], c["T"], B)
        keys = pairs = 0
        for L, n in zip(lens, q_len):  # which length goes with which query count is drawn: the sums hardly depend on it
            first = max(0, L - W + 1)
            keys += L + n - first + min(S, first)
            for t in range(n):
                if c["tree"]:  # a node about t / 9 levels deep sees its few ancestors
                    p, extra = L + t // 9, min(t // 9 + 1, W)
                    lo = max(0, p - W + 1)
                    pairs += max(0, L - lo) + min(S, lo, L) + extra
                else:
                    lo = max(0, L + t - W + 1)
                    pairs += L + t + 1 - lo + min(S, lo)
        rows = sum(q_len) * c["Hq"]
        return {"bytes": keys * row * 2 + rows * (c["D"] * 4 + 4), "flops": 4 * c["D"] * c["Hq"] * pairs}
    if c["op"] == "step":
        B, P = c["B"], -(-(c["hi"] + c["T"]) // PAGE)
        rows = sum(_spread(c["t_lo"], c["T"], B))
        return {"bytes": rows * c["layers"] * c["Hkv"] * c["D"] * 2 * 2 * 2 + B * P * 4, "flops": 0}
    if c["op"] == "fork":
        G, N = c["groups"], c["width"]
        lens = _spread(c["lo"], c["hi"], G)
        # rows that do not keep their parent's last page: all but one, or all but the number of parents drawn
        lost = N - 1 if c["best"] else N * (1 - 1 / N) ** N
        rows = sum((x % PAGE) * lost for x in lens)
        return {"bytes": rows * c["layers"] * c["Hkv"] * c["D"] * 2 * 2 * 2 + G * N * (max(lens) // PAGE + 3) * 8, "flops": 0}
    B, n, r = c["B"], c["n_vis"], c["keep"]
    rows = 0
    for i in range(B):
        L = c["v0"] + n + c["text"] - i * (c["text"] // (2 * B))
        rows += (r + L - c["v0"] - n) if r < n else 0
    return {"bytes": max(4 * B * r, rows * c["layers"] * c["Hkv"] * c["D"] * 2 * 2 * 2), "flops": 0}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The attention from its definition: for each sequence its visible slots, listed one query at a time, in 64 bits.
    The other operators only move values: there is nothing to compute."""
    if case["op"] != "attn":
        return None
    s = prepare(case, seed)
    B, T, Hq, Hkv, D, W, S = (s[x] for x in ("B", "T", "Hq", "Hkv", "D", "window", "sinks"))
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((B, T, Hq), dtype=torch.float64, device=DEV)
    lens, counts = s["kv_len"].tolist(), s["q_len"].tolist()
    for b in range(B):
        L, n = lens[b], counts[b]
        if s["tree"]:
            par = s["parent"][b].tolist()
            depth = _depths(par[:n])
        else:
            depth = list(range(n))
        used = sorted(set(range(max(0, L - W + 1), L + n)) | set(range(min(S, L + n))))
        column = {x: i for i, x in enumerate(used)}
        slot = torch.tensor(used, device=DEV)
        if s["paged"]:
            rows = s["table"][b].long()[slot // PAGE] * PAGE + slot % PAGE
        else:
            rows = slot + b * s["k"].shape[1]
        # committed slots: position = slot; the rest is marked node by node
        mask = torch.zeros((n, len(used)), dtype=torch.bool)
        before = torch.tensor([x for x in used if x < L], dtype=torch.int64)
        for t in range(n):
            p = L + depth[t]
            mask[t, : len(before)] = (p - before < W) | (before < S)
            if s["tree"]:
                a = t
                while a >= 0:
                    mask[t, column[L + a]] = p - (L + depth[a]) < W or L + depth[a] < S
                    a = par[a]
            else:
                new = torch.arange(L, L + n)
                mask[t, len(before):] = (new <= p) & ((p - new < W) | (new < S))
        mask = mask.to(DEV)
        for h in range(Hq):
            k = s["k"].view(-1, Hkv, D)[rows, h // (Hq // Hkv)].double()
            v = s["v"].view(-1, Hkv, D)[rows, h // (Hq // Hkv)].double()
            x = (s["q"][b, :n, h].double() @ k.T) * s["scale"]
            x[~mask] = -math.inf
            lse[b, :n, h] = torch.logsumexp(x, 1)
            out[b, :n, h] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
