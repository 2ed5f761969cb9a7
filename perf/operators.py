"""Measured cases of the block-scaled 8-bit cache: append, attention, eviction.

Each case is one call of one operator on one layer's cache.  With `own` false
the operator is computed in its plain form by elementary torch operations in
fp32 (no fused library calls); with `own` true by the library's kernels.

Cache buffers (one layer):
  codes     int8 or float8_e4m3fn [1][B][H][2][cap][D]   K = 0, V = 1
  scales    float32 [1][B][H][2][cap / 32]
  tail      16-bit  [1][B][H][2][32][D]   tokens of the unfinished block
  positions int32   [1][B][H][cap]
  weights   float32 [1][B][H][cap]        accumulated attention weight
"""
import math

import torch

own = False

DEV = "cuda"
LARGEST = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TINY = 2.0 ** -126

BASE = {"op": "attend", "fmt": "e4m3", "dtype": "bf16", "B": 1, "H": 8, "G": 4, "D": 128,
        "T": 1024, "n": 1, "ragged": False, "strided": False, "gaps": False, "cap": 0.0,
        "window": 0, "slopes": False, "weights": False, "out": "bf16",
        "keep": 0, "sink": 4, "recent": 64}


def _case(**kw):
    return {**BASE, **kw}


def listed():
    return [
        # one decoded token of every sequence of a serving batch: latency
        _case(name="append-int8-token-b16", op="append", fmt="int8", B=16, T=8191, n=1, ragged=True),
        # prompts of one length, K and V as a projection leaves them ([B][n][H][D])
        _case(name="append-e4m3-prompt-b4-t8192", op="append", B=4, T=8192, n=8192, strided=True),
        # padded prompts of several lengths behind a cached prefix, short heads
        _case(name="append-int8-ragged-b7", op="append", fmt="int8", dtype="fp16", B=7, H=4, D=64,
              T=3017, n=1501, ragged=True),
        # one user, short context: the smallest attention call
        _case(name="attend-e4m3-b1-t1024", T=1001, out="fp32"),
        # a serving batch of uneven lengths that keeps the weights for eviction
        _case(name="attend-int8-b16-t8192-weights", fmt="int8", B=16, T=8192, ragged=True, weights=True),
        # large groups, capped scores
        _case(name="attend-e4m3-b4-t32768-cap", B=4, G=8, T=32768, cap=50.0),
        # one user, long context, fp16
        _case(name="attend-int8-b1-t131072", fmt="int8", dtype="fp16", out="fp16", G=8, T=131072),
        # a few drafted tokens checked at once over an evicted cache: window, distance bias
        _case(name="attend-e4m3-b2-n5-window", B=2, H=4, G=3, T=6011, n=5, window=4000, slopes=True,
              gaps=True),
        # whole prompts, capped scores: matrix products
        _case(name="attend-e4m3-prompt-b2-n4096-cap", B=2, T=4096, n=4096, cap=30.0),
        # a prompt's next chunk behind a cached prefix, uneven, with the weights
        _case(name="attend-int8-chunk-b4-n509-weights", fmt="int8", B=4, T=8192, n=509, ragged=True,
              weights=True),
        # a serving batch shrunk to a quarter
        _case(name="evict-int8-b16-t8192", op="evict", fmt="int8", B=16, T=8192, keep=2048, ragged=True),
        # one long context shrunk to an eighth, an odd size
        _case(name="evict-e4m3-b1-t131072", op="evict", T=131071, keep=16001, gaps=True),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    c = dict(BASE)
    c["op"] = rng.choice(["append", "attend", "attend", "evict"])
    c["fmt"] = rng.choice(["int8", "e4m3"])
    c["dtype"] = rng.choice(["bf16", "fp16"])
    c["out"] = c["dtype"]
    c["B"] = _log(rng, 1, 16)
    c["H"] = rng.choice([1, 2, 4, 8])
    c["G"] = rng.choice([1, 2, 3, 4, 6, 8, 16])
    c["D"] = rng.choice([64, 128, 128])
    c["ragged"] = rng.random() < 0.5
    c["gaps"] = rng.random() < 0.3
    heads = c["B"] * c["H"]
    if c["op"] == "append":
        c["n"] = _log(rng, 1, min(8192, 262144 // heads))
        c["T"] = c["n"] + rng.choice([0, _log(rng, 1, 2000)])
        c["strided"] = rng.random() < 0.5
    elif c["op"] == "attend":
        few = rng.random() < 0.6
        c["T"] = _log(rng, 1, min(131072, (1 << 20) // heads)) if few else _log(rng, 32, 4096)
        c["n"] = min(c["T"], _log(rng, 1, 8)) if few else _log(rng, 9, c["T"])
        while heads * c["G"] * c["n"] * c["T"] > 1 << 30:
            c["n"] = max(1, c["n"] // 2)
        c["weights"] = rng.random() < 0.4
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["window"] = rng.choice([0, 0, _log(rng, 1, c["T"])])
        c["slopes"] = rng.random() < 0.3
    else:
        c["T"] = _log(rng, 64, min(131072, (1 << 20) // heads))
        c["keep"] = max(34, int(c["T"] * rng.uniform(0.1, 0.9)))
        c["sink"] = rng.randint(0, 4)
        c["recent"] = rng.randint(1, 30)
    return c


# --------------------------------------------------------------------- inputs
def _lengths(c):
    """Tokens cached before the call and new ones, by sequence."""
    B, T, n = c["B"], c["T"], c["n"]
    if c["op"] == "evict":
        return [max(0, T - (b * T // (2 * B) if c["ragged"] else 0)) for b in range(B)], [0] * B
    past = [T - n if not c["ragged"] else max(0, (T - n) * (B - b) // B - 13 * b) for b in range(B)]
    new = [n if not c["ragged"] or n == 1 else max(1, n - n * b // (2 * B) - b % 3) for b in range(B)]
    return past, new


def _capacity(tokens):
    return (tokens + 31) // 32 * 32 + 32


def _empty(c, cap, dt):
    B, H, D = c["B"], c["H"], c["D"]
    return {"codes": torch.zeros(1, B, H, 2, cap, D, dtype=torch.int8, device=DEV).view(CODE[c["fmt"]]),
            "scales": torch.zeros(1, B, H, 2, cap // 32, device=DEV),
            "tail": torch.zeros(1, B, H, 2, 32, D, dtype=dt, device=DEV),
            "positions": torch.zeros(1, B, H, cap, dtype=torch.int32, device=DEV),
            "weights": torch.zeros(1, B, H, cap, device=DEV)}


def prepare(case, seed):
    """A layer's cache filled up to the call, and the call's inputs.  Keys
    have channels of uneven size (lognormal), as rotated keys do."""
    c = case
    g = torch.Generator(DEV).manual_seed(seed * 2 + 1)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    B, H, D, n, dt = c["B"], c["H"], c["D"], c["n"], DTYPE[c["dtype"]]
    past, new = _lengths(c)
    # an attention call finds the new tokens in the cache already
    held = [p + (w if c["op"] == "attend" else 0) for p, w in zip(past, new)]
    cap = _capacity(max(max(p + w for p, w in zip(past, new)), 1))
    s = {"case": c, "cache": _empty(c, cap, dt),
         "past": torch.tensor(past, dtype=torch.int32, device=DEV),
         "new": torch.tensor(new, dtype=torch.int32, device=DEV)}
    cache = s["cache"]
    channel = torch.exp(randn(1, H, 1, D))
    at = torch.tensor(held, device=DEV)
    if max(held):
        x = randn(B, H, 2, cap, D)
        x[:, :, 0] *= channel
        x = x.to(dt)
        code, scale = _quantize(c["fmt"], x.float().view(B, H, 2, cap // 32, 32 * D))
        cache["codes"][0] = code.view(B, H, 2, cap, D)
        cache["scales"][0] = scale
        row = torch.minimum(at[:, None] // 32 * 32 + torch.arange(32, device=DEV), at.new_tensor(cap - 1))
        cache["tail"][0] = torch.gather(x, 3, row[:, None, None, :, None].expand(B, H, 2, 32, D))
        slot = torch.arange(cap, device=DEV)
        gap = torch.ones(B, H, cap, device=DEV)
        if c["gaps"]:
            jump = torch.rand(B, H, cap, generator=g, device=DEV)
            far = slot < (s["past"][:, None] - 8)[:, None]
            gap += torch.where(far & (jump < 0.2), (jump * 100).floor(), torch.zeros_like(jump))
        pos = torch.cumsum(gap, -1, dtype=torch.float64) - 1
        last = torch.gather(pos, 2, (at - 1).clamp(min=0)[:, None, None].expand(B, H, 1))
        cache["positions"][0] = (pos + last.amax(1, keepdim=True) - last).to(torch.int32)
        # earlier calls' weight: what an evicting call finds, or as much as an attention call adds
        mean = c["G"] * n / c["T"] if c["op"] == "attend" else 1.0
        weight = -mean * torch.log1p(-torch.rand(B, H, cap, generator=g, device=DEV))
        cache["weights"][0] = torch.where(slot < at[:, None, None], weight, torch.zeros_like(weight))
    if c["op"] == "append":
        for name in ("k", "v"):
            x = randn(B, n, H, D) if c["strided"] else randn(B, H, n, D)
            x = x.transpose(1, 2) if c["strided"] else x
            s[name] = (x * channel if name == "k" else x).to(dt)
    elif c["op"] == "attend":
        s["q"] = randn(B, H * c["G"], n, D).to(dt)
        s["out"] = torch.zeros(B, H * c["G"], n, D, dtype=DTYPE[c["out"]], device=DEV)
        s["slopes"] = None
        if c["slopes"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H * c["G"] + 1, device=DEV) / (H * c["G"]))
    else:
        s["to"] = _empty(c, _capacity(c["keep"]), dt)
        s["left"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms
def _quantize(fmt, x):
    """x: fp32 [..][32 D] blocks -> codes and scales [..]."""
    most = LARGEST[fmt]
    scale = x.abs().amax(-1) / most
    scale = torch.where(scale < TINY, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    y = (x * inv[..., None]).clamp(-most, most)
    return (torch.round(y) if fmt == "int8" else y).to(CODE[fmt]), scale


def _values(cache, length, tokens):
    """fp32 [B][H][2][tokens][D] of the first slots, zero from length on."""
    codes, scales, tail = cache["codes"][0], cache["scales"][0], cache["tail"][0]
    B, H, _, _, D = codes.shape
    slot = torch.arange(tokens, device=codes.device)
    full = codes[:, :, :, :tokens].float() * scales.repeat_interleave(32, 3)[:, :, :, :tokens, None]
    rest = tail[:, :, :, slot % 32].float()
    L = length.long()[:, None, None, None, None]
    t = slot[:, None]
    return torch.where(t < L // 32 * 32, full, torch.where(t < L, rest, torch.zeros_like(rest)))


def _append(s):
    c, cache = s["case"], s["cache"]
    B, H, D, n = c["B"], c["H"], c["D"], c["n"]
    past, new = s["past"].long(), s["new"].long()
    total = past + new
    base = past // 32 * 32
    # the blocks the call touches: what the tail holds, then the new rows
    blocks = (31 + n) // 32 + 1
    slot = base[:, None] + torch.arange(blocks * 32, device=DEV)
    row = (slot - past[:, None]).clamp(0, n - 1)[:, None, None, :, None].expand(B, H, 2, -1, D)
    x = torch.gather(torch.stack([s["k"], s["v"]], 2), 3, row)
    old = cache["tail"][0][:, :, :, torch.arange(blocks * 32, device=DEV) % 32]
    held = (slot < past[:, None])[:, None, None, :, None]
    x = torch.where(held, old, x)
    code, scale = _quantize(c["fmt"], x.float().view(B, H, 2, blocks, 32 * D))
    block = torch.arange(blocks, device=DEV) + (base // 32)[:, None]
    cap = cache["codes"].shape[4]
    done = ((block + 1) * 32 <= total[:, None]).view(B, 1, 1, blocks)
    # blocks past the buffer's end are never finished: they land in a spare one
    index = block.clamp(max=cap // 32).view(B, 1, 1, blocks).expand(B, H, 2, -1)
    for name, got, width in (("codes", code.view(torch.int8), 32 * D), ("scales", scale, 1)):
        flat = cache[name][0].view(torch.int8 if width > 1 else torch.float32).view(B, H, 2, cap // 32, width)
        got = got.reshape(B, H, 2, blocks, width)
        wide = torch.cat([flat, flat[:, :, :, :1]], 3)
        where = index[..., None].expand(-1, -1, -1, -1, width)
        wide.scatter_(3, where, torch.where(done[..., None], got, torch.gather(wide, 3, where)))
        flat.copy_(wide[:, :, :, :-1])
    end = total // 32 * 32
    row = (end[:, None] - base[:, None] + torch.arange(32, device=DEV)).clamp(max=blocks * 32 - 1)
    rest = torch.gather(x, 3, row[:, None, None, :, None].expand(B, H, 2, 32, D))
    at = end[:, None] + torch.arange(32, device=DEV)
    fresh = ((at >= past[:, None]) & (at < total[:, None]))[:, None, None, :, None]
    cache["tail"][0] = torch.where(fresh, rest, cache["tail"][0])
    pos, weight = cache["positions"][0], cache["weights"][0]
    last = torch.gather(pos, 2, (past - 1).clamp(min=0)[:, None, None].expand(B, H, 1))
    last = torch.where(past[:, None, None] > 0, last, torch.full_like(last, -1))
    slot = torch.arange(cap, device=DEV)
    mine = ((slot >= past[:, None]) & (slot < total[:, None]))[:, None]
    pos.copy_(torch.where(mine, last + 1 + (slot - past[:, None])[:, None].int(), pos))
    weight.copy_(torch.where(mine, torch.zeros_like(weight), weight))
    return cache


def _attend(s):
    c, cache, q = s["case"], s["cache"], s["q"]
    B, H, G, D, n, T = c["B"], c["H"], c["G"], c["D"], c["n"], c["T"]
    past, new = s["past"].long(), s["new"].long()
    x = _values(cache, past + new, T)
    rows = q.float().reshape(B, H, G * n, D) * (1.0 / math.sqrt(D))
    x = [x[:, :, 0].transpose(2, 3).contiguous(), x[:, :, 1].contiguous()]
    a = torch.matmul(rows, x[0]).view(B, H, G, n, T)
    if c["cap"]:
        a = c["cap"] * torch.tanh(a / c["cap"])
    i, t = torch.arange(n, device=DEV), torch.arange(T, device=DEV)
    at = past[:, None] + i
    pos = cache["positions"][0][:, :, :T].float()
    away = torch.gather(cache["positions"][0], 2, at.clamp(max=cache["positions"].shape[3] - 1)[:, None].expand(B, H, n))
    away = away.float()[..., None] - pos[:, :, None]
    if c["slopes"]:
        a = a - s["slopes"].view(1, H, G, 1, 1) * away[:, :, None]
    seen = (t <= at[..., None]) & (i < new[:, None])[..., None]
    seen = seen[:, None]
    if c["window"]:
        seen = seen & (away < c["window"])
    a = a.masked_fill(~seen[:, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(B, H, G * n, T), x[1]).view(B, H * G, n, D)
    s["out"].copy_(torch.where((i < new[:, None])[:, None, :, None], o, s["out"].float()))
    if not c["weights"]:
        return s["out"]
    cache["weights"][0][:, :, :T] += p.sum((2, 3))
    return s["out"], cache["weights"]


def _evict(s):
    c, cache, to = s["case"], s["cache"], s["to"]
    B, H, D, T, keep = c["B"], c["H"], c["D"], c["T"], c["keep"]
    L = s["past"].long()[:, None, None]
    slot = torch.arange(T, device=DEV)
    weight = cache["weights"][0][:, :, :T]
    rank = torch.where((slot < c["sink"]) | (slot >= L - c["recent"]), torch.full_like(weight, math.inf), weight)
    rank = torch.where(slot < L, rank, torch.full_like(rank, -1.0))
    keep = min(keep, T)
    left = torch.minimum(L, torch.full_like(L, keep))
    kept = torch.sort(rank, stable=True, dim=-1, descending=True)[1][..., :keep]
    nth = torch.arange(keep, device=DEV)
    kept = torch.sort(torch.where(nth < left, kept, torch.full_like(kept, T)), -1)[0]
    kept = kept.clamp(max=T - 1)
    cap = to["codes"].shape[4]
    cover = _capacity(keep)
    wide = torch.cat([kept, kept[..., :1].expand(B, H, cover - keep)], -1)
    x = _values(cache, s["past"], T)
    x = torch.gather(x, 3, wide[:, :, None, :, None].expand(B, H, 2, cover, D))
    code, scale = _quantize(c["fmt"], x.view(B, H, 2, cover // 32, 32 * D))
    done = ((torch.arange(cover // 32, device=DEV) + 1) * 32 <= left)[:, :, None]
    got = torch.where(done[..., None], code.view(torch.int8), torch.zeros_like(code.view(torch.int8)))
    codes = to["codes"][0].view(torch.int8)
    codes[:, :, :, :cover] = torch.where(done[..., None].expand_as(got), got, codes[:, :, :, :cover].reshape(got.shape)).view(B, H, 2, cover, D)
    to["scales"][0][..., :cover // 32] = torch.where(done, scale, to["scales"][0][..., :cover // 32])
    end = left // 32 * 32
    row = end + torch.arange(32, device=DEV)
    rest = torch.gather(x, 3, row.clamp(max=cover - 1)[:, :, None, :, None].expand(B, H, 2, 32, D))
    to["tail"][0] = torch.where((row < left)[:, :, None, :, None], rest.to(to["tail"].dtype), to["tail"][0])
    mine = nth < left
    for name in ("positions", "weights"):
        got = torch.gather(cache[name][0], 2, kept)
        to[name][0][:, :, :keep] = torch.where(mine, got, to[name][0][:, :, :keep])
    s["left"].copy_(left.view(B))
    return to, s["left"]


# ----------------------------------------------------------- the library's own
def _handle(s):
    """The descriptors and the workspace a program makes once for its cache."""
    if "handle" not in s:
        import paper_2605_06675_amd as rq
        c = s["case"]

        def desc(cache):
            return rq.make_block_cache(
                rq.RQ_INT8 if c["fmt"] == "int8" else rq.RQ_E4M3, rq.RQ_BF16 if c["dtype"] == "bf16" else rq.RQ_F16,
                1, c["B"], c["H"], c["H"] * c["G"], c["D"], cache["codes"].shape[4], **cache)

        h = s["handle"] = {"rq": rq, "cache": desc(s["cache"])}
        need = 0
        if c["op"] == "attend":
            need = rq.rq_block_attention_workspace(h["cache"], c["n"], c["T"], c["weights"])
        elif c["op"] == "evict":
            h["to"] = desc(s["to"])
            need = rq.rq_block_evict_workspace(h["cache"], c["keep"])
        h["ws"] = torch.zeros(max(need, 1), dtype=torch.uint8, device=DEV)
        h["new"] = s["new"] if c["ragged"] and c["n"] > 1 else None
    return s["handle"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _append, "attend": _attend, "evict": _evict}[c["op"]](s)
    h = _handle(s)
    rq = h["rq"]
    if c["op"] == "append":
        rq.rq_block_append(h["cache"], 0, s["past"], s["k"], s["v"], new_len=h["new"])
        return s["cache"]
    if c["op"] == "attend":
        rq.rq_block_attention(h["cache"], 0, s["past"], s["q"], s["out"], h["ws"], new_len=h["new"],
                              max_tokens=c["T"], cap=c["cap"], window=c["window"], slopes=s["slopes"],
                              accumulate=c["weights"])
        return (s["out"], s["cache"]["weights"]) if c["weights"] else s["out"]
    rq.rq_block_evict(h["cache"], h["to"], 0, s["past"], c["keep"], s["left"], h["ws"], n_sink=c["sink"],
                      n_recent=c["recent"])
    return s["to"], s["left"]


# ----------------------------------------------------------------- what it costs
def work(case):
    c = case
    past, new = _lengths(c)
    H, G, D = c["H"], c["G"], c["D"]
    if c["op"] == "append":
        rows = sum(new) * H * 2
        coded = sum((p + w) // 32 * 32 - p // 32 * 32 for p, w in zip(past, new)) * H * 2
        return {"bytes": rows * D * 2 + coded * (D + 4 / 32) + sum(new) * H * 8, "flops": 4.0 * rows * D}
    if c["op"] == "evict":
        kept = sum(min(p, c["keep"]) for p in past) * H
        return {"bytes": 4.0 * sum(past) * H + kept * (2 * 2 * (D + 4 / 32) + 16), "flops": 8.0 * kept * D}
    window = c["window"] or 1 << 30
    seen, read = 0, 0
    for p, w in zip(past, new):
        lo = max(0, p + 1 - window)
        read += p + w - lo
        # rows p .. p + w - 1 see min(window, row + 1) tokens
        full = max(0, min(w, p + w + 1 - window))
        short = w - full
        seen += full * min(window, p + w) + short * (p + 1) + short * (short - 1) // 2
    size = 2 if c["out"] != "fp32" else 4
    return {"bytes": read * H * (2 * (D + 4 / 32) + (8 if c["weights"] else 0) + (4 if c["window"] or c["slopes"] else 0))
            + sum(new) * H * G * D * (2 + size),
            "flops": 4.0 * seen * H * G * D}


# ----------------------------------------------------------------- 64-bit results
def _exact_values(c, cache, b, h, L, kind):
    """float64 [L][D] of one head's cached rows."""
    full = L // 32 * 32
    x = cache["codes"][0, b, h, kind, :full].float().double().view(-1, 32, c["D"])
    x = (x * cache["scales"][0, b, h, kind, :full // 32].double().view(-1, 1, 1)).view(full, c["D"])
    return torch.cat([x, cache["tail"][0, b, h, kind, :L - full].double()])


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    cache = s["cache"]
    past, new = _lengths(c)
    B, H, G, D, n = c["B"], c["H"], c["G"], c["D"], c["n"]
    most = LARGEST[c["fmt"]]
    if c["op"] == "append":
        scales = cache["scales"].double()
        for b in range(B):
            p, w = past[b], new[b]
            lo, hi = p // 32 * 32, (p + w) // 32 * 32
            for kind, x in ((0, s["k"]), (1, s["v"])):
                rows = torch.cat([cache["tail"][0, b, :, kind, :p - lo], x[b, :, :w]], 1)[:, :hi - lo]
                if hi > lo:
                    scales[0, b, :, kind, lo // 32:hi // 32] = rows.double().abs().reshape(H, (hi - lo) // 32, -1).amax(-1) / most
        return {"codes": None, "scales": scales, "tail": None, "positions": None, "weights": None}
    if c["op"] == "evict":
        left = torch.tensor([min(p, c["keep"]) for p in past], dtype=torch.int32, device=DEV)
        scales = s["to"]["scales"].double()
        weights = s["to"]["weights"].double()
        for b in range(B):
            for h in range(H):
                L = past[b]
                k = min(L, c["keep"])
                w = cache["weights"][0, b, h, :L].double()
                w[:c["sink"]] = math.inf
                w[max(0, L - c["recent"]):] = math.inf
                bar = torch.topk(w, k)[0][-1] if k else 0.0
                over = torch.nonzero(w > bar).view(-1)
                ties = torch.nonzero(w == bar).view(-1)[:k - over.numel()]
                slots = torch.sort(torch.cat([over, ties]))[0]
                weights[0, b, h, :k] = cache["weights"][0, b, h, slots].double()
                full = k // 32 * 32
                if full:
                    for kind in (0, 1):
                        x = _exact_values(c, cache, b, h, L, kind)[slots[:full]]
                        scales[0, b, h, kind, :full // 32] = x.abs().view(full // 32, -1).amax(-1) / most
        return {"codes": None, "scales": scales, "tail": None, "positions": None, "weights": weights}, left
    out = s["out"].double()
    weights = cache["weights"].double()
    for b in range(B):
        p, w = past[b], new[b]
        L = p + w
        lines = p + torch.arange(w, device=DEV)
        for h in range(H):
            K, V = (_exact_values(c, cache, b, h, L, kind) for kind in (0, 1))
            pos = cache["positions"][0, b, h, :L].double()
            away = pos[lines][:, None] - pos
            hide = torch.arange(L, device=DEV) > lines[:, None]
            if c["window"]:
                hide = hide | (away >= c["window"])
            for g in range(G):
                a = s["q"][b, h * G + g, :w].double() @ K.T / math.sqrt(D)
                if c["cap"]:
                    a = c["cap"] * torch.tanh(a / c["cap"])
                if c["slopes"]:
                    a = a - s["slopes"][h * G + g].double() * away
                a = torch.softmax(a.masked_fill(hide, -math.inf), -1)
                out[b, h * G + g, :w] = a @ V
                if c["weights"]:
                    weights[0, b, h, :L] += a.sum(0)
    return (out, weights) if c["weights"] else out
