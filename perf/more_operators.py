"""Measured cases of speculative decoding over the block-scaled 8-bit cache:
a tree of drafted tokens is laid out (tree), attends over the cache and itself
(attend), is verified against the target's probabilities (verify), and the
accepted path's keys and values are appended to every layer (accept).

With `own` false an operator is computed in its plain form by elementary torch
operations (fp32; fp64 for verification); with `own` true by the library.

Drafted tokens ("nodes") of a sequence are numbered so that a node's parent
comes before it.  parents: int32 [B][n], -1: the last cached token.
  mask   int32 words [B][n][(n + 31) / 32]: bit j % 32 of word j / 32 of row i
         says that node i sees node j (its ancestors and itself)
  depth  int32 [B][n]: ancestors among the nodes
"""
import math
import random

import torch

own = False

DEV = "cuda"
LARGEST = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TINY = 2.0 ** -126

BASE = {"op": "attend", "B": 1, "n": 8, "shape": "tree", "ragged": False,
        # attend, accept: the cache
        "fmt": "e4m3", "dtype": "bf16", "H": 8, "G": 4, "D": 128, "T": 1024, "layers": 1,
        "strided": False, "gaps": False, "cap": 0.0, "window": 0, "slopes": False, "out": "bf16",
        # verify: entries of a row of probabilities, and whether the drafted ones are given
        "V": 32768, "probs": "fp32", "draft": True}


def _case(**kw):
    return {**BASE, **kw}


def listed():
    return [
        # one user, short context, eight drafted tokens of groups of 4: latency
        _case(name="attend-e4m3-b1-n8-t1001", T=1001),
        # a serving batch of uneven lengths, a small tree each: one read of the cache
        _case(name="attend-int8-b16-n7-t8192", fmt="int8", B=16, n=7, T=8192, ragged=True),
        # a serving batch with trees of the usual size: matrix products
        _case(name="attend-e4m3-b8-n64-t8192", B=8, n=64, T=8192, strided=True),
        # one user, long context, a middling tree
        _case(name="attend-int8-b1-n13-t131072", fmt="int8", dtype="fp16", out="fp16", n=13, T=131072),
        # short heads, odd groups, every option, over an evicted cache
        _case(name="attend-e4m3-b5-n21-window-cap", B=5, H=4, G=3, D=64, n=21, T=6011, ragged=True, gaps=True,
              cap=30.0, window=4000, slopes=True, out="fp32"),
        # the usual tree and a very large one, laid out once a step
        _case(name="tree-b16-n64", op="tree", B=16, n=64, ragged=True),
        _case(name="tree-b8-n1000", op="tree", B=8, n=1000, ragged=True),
        # five drafted tokens in a row, drawn from a draft model
        _case(name="verify-chain-b32-n6", op="verify", B=32, n=6, shape="chain"),
        # a tree of several draws a node: a rejected one leaves a residual to the next
        _case(name="verify-tree-b4-n31", op="verify", B=4, n=31, V=100003, ragged=True),
        # trees of a draft model's likeliest tokens, 16-bit probabilities
        _case(name="verify-likeliest-b16-n64", op="verify", B=16, n=64, V=131072, probs="bf16", draft=False),
        # the accepted path in all layers of a model, for a serving batch and for one user
        _case(name="accept-int8-l32-b16-n16", op="accept", fmt="int8", layers=32, B=16, n=16, T=250, ragged=True),
        _case(name="accept-e4m3-l80-b1-n64", op="accept", layers=80, n=64, T=1000, dtype="fp16", strided=True),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    c = dict(BASE)
    c["op"] = rng.choice(["attend", "attend", "attend", "verify", "verify", "accept", "tree"])
    c["shape"] = rng.choice(["tree", "tree", "chain"])
    c["ragged"] = rng.random() < 0.5
    c["B"] = _log(rng, 1, 16)
    if c["op"] == "tree":
        c["n"], c["B"] = _log(rng, 1, 1024), _log(rng, 1, 64)
        return c
    if c["op"] == "verify":
        c["B"], c["n"] = _log(rng, 1, 64), _log(rng, 1, 128)
        c["V"] = _log(rng, 1000, min(131072, (1 << 27) // (c["B"] * c["n"])))
        c["probs"] = rng.choice(["fp32", "fp32", "bf16", "fp16"])
        c["draft"] = rng.random() < 0.6
        return c
    c["fmt"] = rng.choice(["int8", "e4m3"])
    c["dtype"] = rng.choice(["bf16", "fp16"])
    c["out"] = rng.choice([c["dtype"], c["dtype"], "fp32"])
    c["H"] = rng.choice([1, 2, 4, 8])
    c["D"] = rng.choice([64, 128, 128])
    c["strided"] = rng.random() < 0.5
    if c["op"] == "accept":
        c["n"] = _log(rng, 1, 64)
        c["layers"] = _log(rng, 1, 80)
        c["T"] = _log(rng, 1, 1000)
        while c["layers"] * c["B"] * c["H"] * (c["T"] + c["n"] + 64) > 1 << 21:
            c["layers"] = (c["layers"] + 1) // 2
        return c
    c["G"] = rng.choice([1, 2, 3, 4, 6, 8, 16])
    c["n"] = _log(rng, 1, 256)
    heads = c["B"] * c["H"]
    c["T"] = rng.choice([0, 1]) if rng.random() < 0.1 else _log(rng, 1, min(131072, (1 << 20) // heads))
    while heads * c["G"] * c["n"] * c["T"] > 1 << 27:
        if c["n"] > 1:
            c["n"] = (c["n"] + 1) // 2
        else:
            c["T"] //= 2
    c["gaps"] = rng.random() < 0.3
    c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
    c["window"] = rng.choice([0, 0, _log(rng, 1, max(c["T"], 1))])
    c["slopes"] = rng.random() < 0.3
    return c


# --------------------------------------------------------------------- inputs
def _lengths(c):
    """Tokens cached before the call and nodes, by sequence."""
    B, T, n = c["B"], c["T"], c["n"]
    past = [T if not c["ragged"] else max(0, T * (2 * B - b) // (2 * B) - 13 * b) for b in range(B)]
    new = [n if not c["ragged"] else max(1, n - n * b // (2 * B) - b % 3) for b in range(B)]
    return past, new


def _parents(c, seed):
    """[B][n] parents; node 0 is the root.  A tree is wide near the root."""
    rng = random.Random(seed)
    rows = []
    for _ in range(c["B"]):
        row = [-1]
        for i in range(1, c["n"]):
            lo = 0 if c["n"] < 3 else max(0, i // 4 - 2)
            row.append(i - 1 if c["shape"] == "chain" else min(i - 1, rng.randint(lo, max(lo, i // 2))))
        rows.append(row)
    return torch.tensor(rows, dtype=torch.int32, device=DEV)


def _capacity(tokens):
    return (tokens + 31) // 32 * 32 + 32


def _rows(c, g, lead, channel=None):
    """16-bit rows lead + [n][D], as a projection leaves them where strided."""
    n, D, dt = c["n"], c["D"], DTYPE[c["dtype"]]
    if c["strided"]:
        x = torch.randn(*lead[:-1], n, lead[-1], D, generator=g, device=DEV).transpose(-2, -3)
    else:
        x = torch.randn(*lead, n, D, generator=g, device=DEV)
    return (x if channel is None else x * channel).to(dt)


def prepare(case, seed):
    """What a step has in hand: the cache filled up to it and the call's
    inputs.  Keys have channels of uneven size (lognormal), as rotated keys do;
    drafted tokens are drawn from the draft's probabilities (or are its
    likeliest), which are the target's with noise in the logits."""
    c = case
    g = torch.Generator(DEV).manual_seed(seed * 2 + 1)
    B, n = c["B"], c["n"]
    past, new = _lengths(c)
    s = {"case": c, "past": torch.tensor(past, dtype=torch.int32, device=DEV),
         "new": torch.tensor(new, dtype=torch.int32, device=DEV), "parents": _parents(c, seed)}
    if c["op"] == "tree":
        s["mask"] = torch.zeros(B, n, (n + 31) // 32, dtype=torch.int32, device=DEV)
        s["depth"] = torch.zeros(B, n, dtype=torch.int32, device=DEV)
    elif c["op"] == "verify":
        _prepare_verify(s, g)
    else:
        _prepare_cache(s, g, past)
        if c["op"] == "attend":
            channel = torch.exp(torch.randn(1, c["H"], 1, c["D"], generator=g, device=DEV))
            lead = (B, c["H"])
            s["k"], s["v"] = _rows(c, g, lead, channel), _rows(c, g, lead)
            s["q"] = _rows(c, g, (B, c["H"] * c["G"]))
            s["mask"], s["depth"] = _layout(s["parents"])
            s["slopes"] = None
            if c["slopes"]:
                heads = c["H"] * c["G"]
                s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, heads + 1, device=DEV) / heads)
            s["out"] = torch.zeros(B, c["H"] * c["G"], n, c["D"], dtype=DTYPE[c["out"]], device=DEV)
        else:
            lead = (c["layers"], B, c["H"])
            s["k"], s["v"] = _rows(c, g, lead), _rows(c, g, lead)
            rng = random.Random(seed)
            path = torch.full((B, n), -1, dtype=torch.int32)
            count = []
            for b in range(B):
                m = rng.randint(1, max(1, new[b] // 2))
                path[b, :m] = torch.tensor(sorted([0] + rng.sample(range(1, new[b]), m - 1)))
                count.append(m)
            s["path"], s["count"] = path.to(DEV), torch.tensor(count, dtype=torch.int32, device=DEV)
            s["held"] = s["past"].expand(c["layers"], B).contiguous()
            s["lengths"], s["fitting"], s["dropped"] = (torch.zeros_like(s["held"]) for _ in range(3))
    return s


def _prepare_cache(s, g, past):
    c = s["case"]
    L, B, H, D, dt = c["layers"], c["B"], c["H"], c["D"], DTYPE[c["dtype"]]
    cap = _capacity(max(max(past), 1) + (c["n"] if c["op"] == "accept" else 0))
    cache = s["cache"] = {
        "codes": torch.zeros(L, B, H, 2, cap, D, dtype=torch.int8, device=DEV).view(CODE[c["fmt"]]),
        "scales": torch.zeros(L, B, H, 2, cap // 32, device=DEV),
        "tail": torch.zeros(L, B, H, 2, 32, D, dtype=dt, device=DEV),
        "positions": torch.zeros(L, B, H, cap, dtype=torch.int32, device=DEV)}
    at = s["past"]
    slot = torch.arange(cap, device=DEV)
    gap = torch.ones(L, B, H, cap, device=DEV)
    if c["gaps"]:
        jump = torch.rand(L, B, H, cap, generator=g, device=DEV)
        far = slot < (at[:, None] - 8)[:, None]
        gap += torch.where(far & (jump < 0.2), (jump * 100).floor(), torch.zeros_like(jump))
    cache["positions"].copy_(torch.cumsum(gap, -1, dtype=torch.float64) - 1)
    if not max(past):
        return
    row = torch.minimum(at[:, None] // 32 * 32 + torch.arange(32, device=DEV), at.new_tensor(cap - 1))
    channel = torch.exp(torch.randn(1, H, 1, D, generator=g, device=DEV))
    for layer in range(L):
        x = torch.randn(B, H, 2, cap, D, generator=g, device=DEV)
        x[:, :, 0] *= channel
        x = x.to(dt)
        code, scale = _quantize(c["fmt"], x.float().view(B, H, 2, cap // 32, 32 * D))
        cache["codes"][layer] = code.view(B, H, 2, cap, D)
        cache["scales"][layer] = scale
        cache["tail"][layer] = torch.gather(x, 3, row[:, None, None, :, None].expand(B, H, 2, 32, D))


def _prepare_verify(s, g):
    c = s["case"]
    B, n, V, dt = c["B"], c["n"], c["V"], DTYPE[c["probs"]]
    parents = s["parents"].long()
    target = torch.empty(B, n, V, dtype=dt, device=DEV)
    draft = torch.empty(B, n, V, dtype=dt, device=DEV)
    tokens = torch.randint(V, (B, n), generator=g, device=DEV)
    rows = torch.arange(B, device=DEV)
    # which of its siblings a node is
    nth = (torch.tril(parents[:, :, None] == parents[:, None], -1)).sum(-1)
    for i in range(n):
        x = 2.5 * torch.randn(B, V, generator=g, device=DEV)
        target[:, i] = torch.softmax(x, -1).to(dt)
        draft[:, i] = torch.softmax(x + 0.7 * torch.randn(B, V, generator=g, device=DEV), -1).to(dt)
        if i == 0:
            continue
        p = draft[rows, parents[:, i]].float()
        if c["draft"]:
            noise = -torch.log(-torch.log(torch.rand(B, V, generator=g, device=DEV).clamp(1e-12, 1 - 1e-7)))
            tokens[:, i] = (torch.log(p) + noise).argmax(-1)
        else:
            best = p.topk(min(V, int(nth[:, i].max()) + 1), -1)[1]
            tokens[:, i] = best[rows, nth[:, i]]
    s["target"], s["draft"] = target, draft if c["draft"] else None
    s["tokens"] = tokens.int()
    s["uniforms"] = torch.rand(B, n, generator=g, device=DEV)
    s["path"] = torch.zeros(B, n, dtype=torch.int32, device=DEV)
    s["count"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    s["next"] = torch.zeros(B, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------- plain forms
def _quantize(fmt, x):
    """x: fp32 [..][32 D] blocks -> codes and scales [..]."""
    most = LARGEST[fmt]
    scale = x.abs().amax(-1) / most
    scale = torch.where(scale < TINY, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    y = (x * inv[..., None]).clamp(-most, most)
    return (torch.round(y) if fmt == "int8" else y).to(CODE[fmt]), scale


def _layout(parents):
    """Mask words and depths of [B][n] parents: the closure of the parent
    relation by repeated squaring."""
    B, n = parents.shape
    node = torch.arange(n, device=parents.device)
    sees = ((parents[:, :, None] == node) | (node[:, None] == node)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        sees = (torch.matmul(sees, sees) > 0).float()
    depth = sees.sum(-1).int() - 1
    words = (n + 31) // 32
    bits = torch.zeros(B, n, words * 32, dtype=torch.int64, device=parents.device)
    bits[:, :, :n] = sees.long()
    word = (bits.view(B, n, words, 32) << torch.arange(32, device=parents.device)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int(), depth


def _tree(s):
    mask, depth = _layout(s["parents"])
    mine = (torch.arange(s["case"]["n"], device=DEV) < s["new"][:, None])
    s["mask"].copy_(torch.where(mine[..., None], mask, s["mask"]))
    s["depth"].copy_(torch.where(mine, depth, s["depth"]))
    return s["mask"], s["depth"]


def _sees(s):
    """bool [B][n][n]."""
    n = s["case"]["n"]
    j = torch.arange(n, device=DEV)
    return (s["mask"][:, :, j // 32] >> (j % 32) & 1).bool()


def _attend(s):
    c, cache = s["case"], s["cache"]
    B, H, G, D, n, T = c["B"], c["H"], c["G"], c["D"], c["n"], c["T"]
    past, new = s["past"].long(), s["new"].long()
    slot = torch.arange(T, device=DEV)
    codes, scales, tail = cache["codes"][0], cache["scales"][0], cache["tail"][0]
    full = codes[:, :, :, :T].float() * scales.repeat_interleave(32, 3)[:, :, :, :T, None]
    at = past[:, None, None, None, None]
    x = torch.where(slot[:, None] < at // 32 * 32, full, tail[:, :, :, slot % 32].float())
    x = torch.where(slot[:, None] < at, x, torch.zeros_like(x))
    i = torch.arange(n, device=DEV)
    own_rows = (i < new[:, None])[:, None, :, None]
    k = torch.cat([x[:, :, 0], torch.where(own_rows, s["k"], torch.zeros_like(s["k"])).float()], 2)
    v = torch.cat([x[:, :, 1], torch.where(own_rows, s["v"], torch.zeros_like(s["v"])).float()], 2)
    rows = s["q"].float().reshape(B, H, G * n, D) * (1.0 / math.sqrt(D))
    a = torch.matmul(rows, k.transpose(2, 3).contiguous()).view(B, H, G, n, T + n)
    if c["cap"]:
        a = c["cap"] * torch.tanh(a / c["cap"])
    last = torch.gather(cache["positions"][0], 2, (past - 1).clamp(min=0)[:, None, None].expand(B, H, 1))
    last = torch.where(past[:, None, None] > 0, last, torch.full_like(last, -1)).long()
    mine = last + 1 + s["depth"][:, None]
    pos = torch.cat([cache["positions"][0][:, :, :T].long(), mine], 2)
    away = (mine[..., None] - pos[:, :, None]).float()
    if c["slopes"]:
        a = a - s["slopes"].view(1, H, G, 1, 1) * away[:, :, None]
    seen = torch.cat([(slot < past[:, None])[:, None].expand(B, n, T), _sees(s) & (i < new[:, None])[:, None]], 2)
    seen = (seen & (i < new[:, None])[..., None])[:, None]
    if c["window"]:
        seen = seen & (away < c["window"])
    a = a.masked_fill(~seen[:, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(B, H, G * n, T + n), v).view(B, H * G, n, D)
    s["out"].copy_(torch.where((i < new[:, None])[:, None, :, None], o, s["out"].float()))
    return s["out"]


def _verify(s):
    c = s["case"]
    B, n, V = c["B"], c["n"], c["V"]
    target, draft = s["target"], s["draft"]
    rows = torch.arange(B, device=DEV)
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    path = torch.full((B, n), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    count = torch.ones(B, dtype=torch.int32, device=DEV)
    r = target[:, 0].double()
    mass = torch.ones(B, dtype=torch.float64, device=DEV)
    # a node is looked at where its parent is the last accepted one by then
    for i in range(1, n):
        mine = (s["parents"][:, i] == cur) & (i < s["new"])
        x = s["tokens"][:, i].long()
        rx = r[rows, x]
        chance = s["uniforms"][:, i].double()
        if draft is not None:
            q = draft[rows, cur].double()
            chance = chance * q[rows, x]
        yes = mine & (chance * mass < rx)
        no = mine & ~yes
        if draft is not None:
            left = (r / torch.where(mass > 0, mass, torch.ones_like(mass))[:, None] - q).clamp(min=0)
            r = torch.where(no[:, None], left, r)
            mass = torch.where(no, left.sum(-1), mass)
        else:
            mass = torch.where(no, (mass - rx).clamp(min=0), mass)
            r[rows, x] = torch.where(no, torch.zeros_like(rx), rx)
        r = torch.where(yes[:, None], target[:, i].double(), r)
        mass = torch.where(yes, torch.ones_like(mass), mass)
        cur = torch.where(yes, torch.full_like(cur, i), cur)
        at = count.long().clamp(max=n - 1)
        path[rows, at] = torch.where(yes, torch.full_like(path[:, 0], i), path[rows, at])
        count = count + yes.int()
    r = torch.where(r.sum(-1, keepdim=True) > 0, r, target[rows, cur].double())
    cum = torch.cumsum(r, -1)
    first = (cum <= s["uniforms"][:, :1].double() * cum[:, -1:]).sum(-1)
    last = (torch.arange(1, V + 1, device=DEV) * (r > 0)).amax(-1) - 1
    s["path"].copy_(path)
    s["count"].copy_(count)
    s["next"].copy_(torch.minimum(first, last).clamp(min=0))
    return s["path"], s["count"], s["next"]


def _accept(s):
    c, cache = s["case"], s["cache"]
    L, B, H, D, n = c["layers"], c["B"], c["H"], c["D"], c["n"]
    cap = cache["codes"].shape[4]
    past = s["held"].long()
    new = torch.minimum(s["count"].long().expand(L, B), cap - past)
    total, base = past + new, past // 32 * 32
    blocks = (31 + n) // 32 + 1
    slot = base[..., None] + torch.arange(blocks * 32, device=DEV)
    nth = (slot - past[..., None]).clamp(0, n - 1)
    node = torch.gather(s["path"].long().expand(L, B, n), 2, nth).clamp(min=0)
    x = torch.stack([s["k"], s["v"]], 3)
    x = torch.gather(x, 4, node[:, :, None, None, :, None].expand(L, B, H, 2, -1, D))
    old = cache["tail"][:, :, :, :, torch.arange(blocks * 32, device=DEV) % 32]
    x = torch.where((slot < past[..., None])[:, :, None, None, :, None], old, x)
    code, scale = _quantize(c["fmt"], x.float().view(L, B, H, 2, blocks, 32 * D))
    block = torch.arange(blocks, device=DEV) + (base // 32)[..., None]
    done = ((block + 1) * 32 <= total[..., None])[:, :, None, None]
    # blocks past the buffer's end are never finished: they land in a spare one
    index = block.clamp(max=cap // 32)[:, :, None, None].expand(L, B, H, 2, blocks)
    for name, got, width in (("codes", code.view(torch.int8), 32 * D), ("scales", scale, 1)):
        flat = cache[name].view(torch.int8 if width > 1 else torch.float32).view(L, B, H, 2, cap // 32, width)
        wide = torch.cat([flat, flat[:, :, :, :, :1]], 4)
        where = index[..., None].expand(-1, -1, -1, -1, -1, width)
        got = torch.where(done[..., None], got.reshape(L, B, H, 2, blocks, width), torch.gather(wide, 4, where))
        wide.scatter_(4, where, got)
        flat.copy_(wide[:, :, :, :, :-1])
    end = total // 32 * 32
    row = (end[..., None] - base[..., None] + torch.arange(32, device=DEV)).clamp(max=blocks * 32 - 1)
    rest = torch.gather(x, 4, row[:, :, None, None, :, None].expand(L, B, H, 2, 32, D))
    at = end[..., None] + torch.arange(32, device=DEV)
    fresh = ((at >= past[..., None]) & (at < total[..., None]))[:, :, None, None, :, None]
    cache["tail"].copy_(torch.where(fresh, rest, cache["tail"]))
    pos = cache["positions"]
    last = torch.gather(pos, 3, (past - 1).clamp(min=0)[..., None, None].expand(L, B, H, 1))
    last = torch.where(past[..., None, None] > 0, last, torch.full_like(last, -1))
    slot = torch.arange(cap, device=DEV)
    mine = ((slot >= past[..., None]) & (slot < total[..., None]))[:, :, None]
    pos.copy_(torch.where(mine, last + 1 + (slot - past[..., None])[:, :, None].int(), pos))
    s["lengths"].copy_(total)
    s["fitting"].copy_(new)
    s["dropped"].copy_(s["count"] - new)
    return cache, s["lengths"], s["fitting"], s["dropped"]


# ----------------------------------------------------------- the library's own
def _handle(s):
    """The descriptor and the workspace that a program makes once."""
    if "handle" not in s:
        import paper_2605_06675_amd as rq
        c = s["case"]
        h = s["handle"] = {"rq": rq, "new": s["new"] if c["ragged"] else None}
        need = 0
        if c["op"] == "verify":
            need = rq.rq_tree_verify_workspace(c["B"], c["n"], c["V"])
        elif c["op"] != "tree":
            h["cache"] = rq.make_block_cache(
                rq.RQ_INT8 if c["fmt"] == "int8" else rq.RQ_E4M3, rq.RQ_BF16 if c["dtype"] == "bf16" else rq.RQ_F16,
                c["layers"], c["B"], c["H"], c["H"] * c["G"], c["D"], s["cache"]["codes"].shape[4], **s["cache"])
            if c["op"] == "attend":
                need = rq.rq_block_tree_attention_workspace(h["cache"], c["n"], c["T"], c["window"])
        h["ws"] = torch.zeros(max(need, 1), dtype=torch.uint8, device=DEV)
    return s["handle"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"attend": _attend, "tree": _tree, "verify": _verify, "accept": _accept}[c["op"]](s)
    h = _handle(s)
    rq = h["rq"]
    if c["op"] == "tree":
        rq.rq_tree_mask(s["parents"], s["mask"], s["depth"], new_len=h["new"])
        return s["mask"], s["depth"]
    if c["op"] == "attend":
        rq.rq_block_tree_attention(h["cache"], 0, s["past"], s["q"], s["k"], s["v"], s["mask"], s["out"], h["ws"],
                                   depth=s["depth"], new_len=h["new"], max_tokens=c["T"], cap=c["cap"],
                                   window=c["window"], slopes=s["slopes"])
        return s["out"]
    if c["op"] == "verify":
        rq.rq_tree_verify(s["tokens"], s["parents"], s["target"], s["draft"], s["uniforms"], s["path"], s["count"],
                          s["next"], h["ws"], new_len=h["new"])
        return s["path"], s["count"], s["next"]
    rq.rq_block_accept(h["cache"], s["held"], s["path"], s["count"], s["k"], s["v"], s["lengths"],
                       fitting=s["fitting"], dropped=s["dropped"])
    return s["cache"], s["lengths"], s["fitting"], s["dropped"]


# ----------------------------------------------------------------- what it costs
def work(case):
    c = case
    past, new = _lengths(c)
    B, H, G, D, n = c["B"], c["H"], c["G"], c["D"], c["n"]
    if c["op"] == "tree":
        return {"bytes": sum(new) * (8 + 4 * ((n + 31) // 32)), "flops": 1.0 * sum(m * m for m in new)}
    if c["op"] == "verify":
        # every node's token, parent, random number and probabilities, and the
        # row (two with a draft) that the last token is drawn from
        size, sides = (4 if c["probs"] == "fp32" else 2), (2 if c["draft"] else 1)
        return {"bytes": sum(new) * (12 + size * sides) + B * (c["V"] * size * sides + 4 * n + 8),
                "flops": 3.0 * B * c["V"]}
    if c["op"] == "accept":
        rows = c["layers"] * H * 2 * sum(max(1, m // 4) for m in new)
        return {"bytes": rows * (D * 4 + 4), "flops": 4.0 * rows * D}
    read = seen = 0
    for p, m in zip(past, new):
        held = min(p, c["window"]) if c["window"] else p
        read += held
        seen += m * (held + m)
    size = 2 if c["out"] != "fp32" else 4
    return {"bytes": read * H * (2 * (D + 4 / 32) + (4 if c["window"] or c["slopes"] else 0))
            + sum(new) * (H * 2 * D * 2 + H * G * D * (2 + size)),
            "flops": 4.0 * seen * H * G * D}


# ----------------------------------------------------------------- 64-bit results
def _exact_rows(c, cache, layer, b, h, L, kind):
    """float64 [L][D] of one head's cached rows."""
    full = L // 32 * 32
    x = cache["codes"][layer, b, h, kind, :full].float().double().view(-1, 32, c["D"])
    x = (x * cache["scales"][layer, b, h, kind, :full // 32].double().view(-1, 1, 1)).view(full, c["D"])
    return torch.cat([x, cache["tail"][layer, b, h, kind, :L - full].double()])


def _chains(parents):
    """For every node the list of its ancestors and itself."""
    chains = []
    for i, p in enumerate(parents):
        chains.append((chains[p] if p >= 0 else []) + [i])
    return chains


def _exact_tree(c, s):
    mask, depth = s["mask"].cpu().clone(), s["depth"].cpu().clone()
    for b, (row, m) in enumerate(zip(s["parents"].tolist(), _lengths(c)[1])):
        for i, chain in enumerate(_chains(row)[:m]):
            depth[b, i] = len(chain) - 1
            words = [0] * mask.shape[2]
            for j in chain:
                words[j // 32] |= 1 << (j % 32)
            mask[b, i] = torch.tensor([w - (w >> 31 << 32) for w in words], dtype=torch.int32)
    return mask, depth


def _exact_verify(c, s):
    paths, counts, nexts = [], [], []
    for b, m in enumerate(_lengths(c)[1]):
        parents, tokens = s["parents"][b, :m].tolist(), s["tokens"][b, :m].tolist()
        u = s["uniforms"][b].double().tolist()
        walk, going = [0], True
        while going:
            at, going = walk[-1], False
            r, mass = s["target"][b, at].double(), 1.0
            for child in [i for i in range(1, m) if parents[i] == at]:
                x = tokens[child]
                q = s["draft"][b, at].double() if c["draft"] else None
                if u[child] * (float(q[x]) if c["draft"] else 1.0) * mass < float(r[x]):
                    walk.append(child)
                    going = True
                    break
                if c["draft"]:
                    r = torch.relu(r / mass - q) if mass > 0 else r * 0
                    mass = float(r.sum())
                else:
                    mass = max(0.0, mass - float(r[x]))
                    r = r.clone()
                    r[x] = 0
        if not float(r.sum()) > 0:
            r = s["target"][b, walk[-1]].double()
        edge = torch.cumsum(r, 0)
        over = torch.nonzero(edge > u[0] * edge[-1])
        paths.append(walk + [-1] * (c["n"] - len(walk)))
        counts.append(len(walk))
        nexts.append(int(over[0] if over.numel() else torch.nonzero(r > 0)[-1]))
    return tuple(torch.tensor(x, dtype=torch.int32) for x in (paths, counts, nexts))


def _exact_accept(c, s):
    scales = s["cache"]["scales"].double()
    fits = s["count"].cpu().tolist()
    for b, (p, m) in enumerate(zip(_lengths(c)[0], fits)):
        nodes = s["path"][b, :m].long()
        lo, hi = p // 32 * 32, (p + m) // 32 * 32
        for kind, x in ((0, s["k"]), (1, s["v"])):
            rows = torch.cat([s["cache"]["tail"][:, b, :, kind, :p - lo], x[:, b][:, :, nodes]], 2)[:, :, :hi - lo]
            if hi > lo:
                most = rows.double().abs().reshape(c["layers"], c["H"], (hi - lo) // 32, -1).amax(-1)
                scales[:, b, :, kind, lo // 32:hi // 32] = most / LARGEST[c["fmt"]]
    fitting = s["count"].expand(c["layers"], c["B"]).contiguous()
    return ({"codes": None, "scales": scales, "tail": None, "positions": None}, s["held"] + fitting, fitting,
            torch.zeros_like(fitting))


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] != "attend":
        return {"tree": _exact_tree, "verify": _exact_verify, "accept": _exact_accept}[c["op"]](c, s)
    out = s["out"].double()
    H, G, D = c["H"], c["G"], c["D"]
    parents = s["parents"].tolist()
    for b, (p, m) in enumerate(zip(*_lengths(c))):
        chains = _chains(parents[b][:m])
        sees = torch.zeros(m, m, dtype=torch.bool)
        for i, chain in enumerate(chains):
            sees[i, chain] = True
        hide = torch.cat([torch.zeros(m, p, dtype=torch.bool), ~sees], 1).to(DEV)
        deep = torch.tensor([len(x) - 1 for x in chains], dtype=torch.float64, device=DEV)
        for h in range(H):
            K, V = (torch.cat([_exact_rows(c, s["cache"], 0, b, h, p, kind), x[b, h, :m].double()])
                    for kind, x in ((0, s["k"]), (1, s["v"])))
            held = s["cache"]["positions"][0, b, h, :p].double()
            here = (held[-1] if p else held.new_tensor(-1.0)) + 1 + deep
            away = here[:, None] - torch.cat([held, here])
            shut = hide | (away >= c["window"]) if c["window"] else hide
            for j in range(h * G, h * G + G):
                a = s["q"][b, j, :m].double() @ K.T.contiguous() / math.sqrt(D)
                if c["cap"]:
                    a = c["cap"] * torch.tanh(a / c["cap"])
                if c["slopes"]:
                    a = a - s["slopes"][j].double() * away
                out[b, j, :m] = torch.softmax(a.masked_fill(shut, -math.inf), -1) @ V
    return out
