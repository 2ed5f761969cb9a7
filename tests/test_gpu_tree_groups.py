"""Tree attention of more than 16 query rows: each kernel that its plan chooses (groups
of 32 or 64 rows, workgroups of four or eight waves, one split or several), which one a
call launched read from the call as a stream capture records it.

Bounds: those of test_gpu_tree."""
import ctypes as C
import math
import re

import numpy as np
import pytest
import torch

import paper_2605_06675_amd as rq
from oracle import tree
from test_gpu_block import DT, FMT, both, ints, types
from test_gpu_tree import Trees, some_parents

pytestmark = pytest.mark.gpu


class KernelParams(C.Structure):
    _fields_ = [("block", C.c_uint32 * 3), ("extra", C.c_void_p), ("func", C.c_void_p),
                ("grid", C.c_uint32 * 3), ("params", C.c_void_p), ("shared", C.c_uint32)]


def launches(call):
    """(name, grid, block) of the kernels that call(stream) launches; none runs."""
    L, stream = rq.lib(), torch.cuda.Stream()
    L.hipKernelNameRefByPtr.restype = C.c_char_p
    graph, n = C.c_void_p(), C.c_size_t()
    assert L.hipStreamBeginCapture(C.c_void_p(stream.cuda_stream), 2) == 0
    try:
        call(stream)
    finally:
        assert L.hipStreamEndCapture(C.c_void_p(stream.cuda_stream), C.byref(graph)) == 0
    assert L.hipGraphGetNodes(graph, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert L.hipGraphGetNodes(graph, nodes, C.byref(n)) == 0
    out = []
    for node in nodes:
        p = KernelParams()
        assert L.hipGraphKernelNodeGetParams(C.c_void_p(node), C.byref(p)) == 0
        name = L.hipKernelNameRefByPtr(C.c_void_p(p.func), C.c_void_p(stream.cuda_stream))
        out.append((name.decode(), tuple(p.grid), tuple(p.block)))
    assert L.hipGraphDestroy(graph) == 0
    return out


def attend_at_once(unit, k, v, seen, depth, q, scale, cap=0.0, window=0, slopes=None, at="cuda"):
    """tree.attend with all rows of a unit together; also a row's largest sum of
    |scale q k|, and that with the largest |q| or the largest |k| in place of each."""
    K, V = (torch.from_numpy(np.concatenate([unit.values(i), x]).astype(np.float64)).to(at) for i, x in ((0, k), (1, v)))
    q = torch.from_numpy(np.ascontiguousarray(q, np.float64)).to(at)
    m, G, D = q.shape
    first = int(unit.pos[-1]) + 1 if unit.length else 0
    own = first + np.asarray(depth, np.int64)
    away = torch.from_numpy((own[:, None] - np.concatenate([unit.pos, own])[None]).astype(np.float64)).to(at)
    sees = torch.from_numpy(np.concatenate([np.ones((m, unit.length), bool), np.asarray(seen, bool)], 1)).to(at)
    if window:
        sees &= away < window
    keys = K.T.contiguous()
    x = scale * (q.view(m * G, D) @ keys).view(m, G, -1)
    if cap:
        x = cap * torch.tanh(x / cap)
    if slopes is not None:
        x = x - torch.tensor(np.asarray(slopes), dtype=torch.float64, device=at)[:, None] * away[:, None]
    x = x.masked_fill(~sees[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = (p.view(m * G, -1) @ V).view(m, G, D) / torch.where(total == 0, torch.ones_like(total), total)
    aq, ak = q.abs(), keys.abs()
    a = abs(scale) * (aq.view(m * G, D) @ ak).amax(-1).view(m, G)
    a2 = abs(scale) * torch.maximum(aq.amax(-1) * ak.sum(0).amax(), aq.sum(-1) * ak.amax())
    return o.cpu().numpy(), a.cpu().numpy(), a2.cpu().numpy(), float(V.abs().max())


class Held:
    """What the oracle asks of a unit's cached tokens."""

    def __init__(self, K, V, pos):
        self.x, self.pos, self.length = (K, V), pos, len(pos)

    def values(self, kind):
        return self.x[kind]


class Filled(Trees):
    """A cache of one layer filled with codes, scales and rows as they come, positions
    with gaps; unused memory holds NaNs."""

    def __init__(self, fmt, dtype, B, H, G, D, held, seed=0):
        self.fmt, self.B, self.H, self.G, self.D, self.layer = fmt, B, H, G, D, 0
        self.rdt, self.dt = DT[dtype]
        self.cap = (max(held) + 31) // 32 * 32 + 32
        self.g = torch.Generator().manual_seed(seed)
        self.channel = torch.exp(0.5 * torch.randn(H, 1, D, generator=self.g))
        c = self.c = rq.BlockCache(FMT[fmt][0], self.rdt, 1, B, H, H * G, D, self.cap)
        codes = torch.randint(0, 256, (B, H, 2, self.cap, D), generator=self.g, dtype=torch.uint8)
        if fmt == "int8":
            codes[codes == 128] = 0                      # (-128 is no code)
        else:
            codes[codes & 0x7f > 0x6f] ^= 0x70           # (small ones are frequent, none is NaN)
        scales = (0.3 + torch.rand(B, H, 2, self.cap // 32, generator=self.g)) / 64
        tail = torch.randn(B, H, 2, 32, D, generator=self.g).to(self.dt)
        gaps = torch.randint(1, 40, (B, H, self.cap), generator=self.g)
        gaps[torch.rand(B, H, self.cap, generator=self.g) < 0.8] = 1
        pos = (gaps.cumsum(-1) - 1).int()
        at, slot = torch.tensor(held)[:, None], torch.arange(self.cap)
        done = (slot < at // 32 * 32)[:, None, None]
        value = codes.view(torch.int8).double() if fmt == "int8" else codes.view(torch.float8_e4m3fn).double()
        value = (value * scales.double().repeat_interleave(32, 3)[..., None]).numpy()
        codes[~done.expand(B, H, 2, self.cap)] = 0x7f
        scales[~done[..., ::32].expand(B, H, 2, self.cap // 32)] = math.nan
        tail[(torch.arange(32) >= at % 32)[:, None, None].expand(B, H, 2, 32)] = math.nan
        pos[(slot >= at)[:, None].expand(B, H, self.cap)] = -(1 << 30)
        self.u = []
        for b, n in enumerate(held):
            x = [[np.concatenate([value[b, h, i, :n // 32 * 32], tail[b, h, i, :n % 32].float().numpy()]) for i in (0, 1)]
                 for h in range(H)]
            self.u.append([Held(*x[h], pos[b, h, :n].numpy()) for h in range(H)])
        c.codes.copy_(codes.view(-1))
        c.scales.copy_(scales.view(-1))
        c.tail.copy_(tail.view(-1))
        c.positions.copy_(pos.view(-1))
        c.lengths.copy_(ints([held]))
        c.bound = [max(held)]


    def compare_tree(self, o, q, k, v, m, seen, depth, scale=None, cap=0.0, window=0, slopes=None):
        """As Trees has it."""
        G, D = self.G, self.D
        scale = D ** -0.5 if scale is None else scale
        half = 0.0 if o.dtype == torch.float32 else torch.finfo(o.dtype).eps / 2
        tiny = 2.0 ** -25 if o.dtype == torch.float16 else 1e-30
        o = o.cpu().double().numpy()
        assert np.isfinite(o).all()
        for b in range(self.B):
            assert (o[b, :, m[b]:] == 7.5).all()
            for h in range(self.H if m[b] else 0):
                u = self.u[b][h]
                kk, vv = (x[b, h, :m[b]].float().numpy() for x in (k, v))
                qq = q[b, h * G:(h + 1) * G, :m[b]].float().numpy().transpose(1, 0, 2)
                sl = None if slopes is None else slopes[h * G:(h + 1) * G]
                want, a, a2, most = attend_at_once(u, kk, vv, seen[b], depth[b], qq, scale, cap, window, sl)
                far = 0.0 if sl is None else 1.4427 * max(sl) * (float(u.pos.max()) if u.length else 0.0) + 64
                s = 1.4427 * (D * 2.0 ** -24 * a + (2 * D * 2.0 ** -25 * a2 if self.dt == torch.bfloat16 else 0))
                s = s + 4 * 2.0 ** -24 * (1.4427 * a + far) + (1.4427 * cap * 2.0 ** -21 if cap else 0)
                ratio = 2 * s * math.log(2) + 2.0 ** -21 + ((u.length + m[b]) / 4 + 64) * 2.0 ** -24
                got = o[b, h * G:(h + 1) * G, :m[b]].transpose(1, 0, 2)
                err = np.abs(got - want) / ((ratio[..., None] + 2.0 ** -21) * most + half * np.abs(want) + tiny)
                assert (err <= 1).all(), (b, h, float(err.max()))


def launched_kernel(r, n, **kw):
    """(rows of a group, waves, splits, options) of a call's first kernel."""
    B, H, G, D = r.B, r.H, r.G, r.D
    held = r.lengths()
    x = torch.zeros(B, H * G, n, D, dtype=r.dt, device="cuda")
    words = torch.zeros(B, n, (n + 31) // 32, dtype=torch.int32, device="cuda")
    ws = torch.zeros(max(16, rq.rq_block_tree_attention_workspace(r.c.desc, n, max(held), kw.get("window", 0))),
                     dtype=torch.uint8, device="cuda")
    past, depth = ints(held), torch.zeros(B, n, dtype=torch.int32, device="cuda")
    if "slopes" in kw:
        kw["slopes"] = torch.tensor(kw["slopes"]).cuda()
    torch.cuda.synchronize()
    found = launches(lambda s: rq.rq_block_tree_attention(
        r.c.desc, 0, past, x, x[:, :H], x[:, :H], words, x, ws, depth=depth, max_tokens=max(held), stream=s, **kw))
    name, grid, block = found[0]
    fmt, d, bf16, tiles, waves, plain = map(int, re.search(r"tree_rows_kernelILi(\d)ELi(\d+)ELb(\d)ELi(\d)ELi(\d)ELb(\d)E",
                                                           name).groups())
    assert (fmt, d, bf16) == (FMT[r.fmt][0], D, r.dt == torch.bfloat16) and block == (64 * waves, 1, 1)
    groups = (n * G + 32 * tiles - 1) // (32 * tiles)
    assert grid[0] % (groups * B * H) == 0 and grid[1:] == (1, 1)
    splits = grid[0] // (groups * B * H)
    assert len(found) == 1 + (splits > 1)
    return 32 * tiles, waves, splits, not plain


SETS = [  # D, rows of a group, waves, splits; B, H, G, n, T
    (64, 32, 4, 1, 1, 1, 6, 3, 8), (64, 32, 4, 17, 2, 3, 3, 43, 2012),
    (64, 32, 8, 1, 2, 1, 5, 4, 100), (64, 32, 8, 6, 1, 1, 1, 17, 1260),
    (64, 64, 4, 1, 24, 8, 6, 11, 9), (64, 64, 4, 3, 2, 4, 6, 174, 3141),
    (64, 64, 8, 1, 12, 2, 3, 108, 2843), (64, 64, 8, 3, 12, 1, 5, 65, 8907),
    (128, 32, 4, 1, 1, 1, 6, 3, 8), (128, 32, 4, 11, 3, 3, 1, 132, 1164),
    (128, 32, 8, 1, 2, 1, 5, 4, 100), (128, 32, 8, 4, 2, 1, 5, 4, 740),
    (128, 64, 4, 1, 24, 8, 6, 11, 9), (128, 64, 4, 3, 2, 4, 5, 206, 2337),
    (128, 64, 8, 1, 3, 2, 6, 226, 1206), (128, 64, 8, 3, 3, 1, 8, 174, 4132)]


@both
@types
@pytest.mark.parametrize("kind", SETS, ids=lambda k: "-".join(map(str, k)))
def test_groups_waves_and_splits(fmt, dtype, kind):
    """Without options, then with all of them (64 rows of 128 channels have no kernel for
    these: the plan takes 32), all nodes and a ragged batch, the last group not full."""
    D, rows, waves, splits, B, H, G, n, T = kind
    held = [max(0, T - 37 * b) for b in range(B)]
    r = Filled(fmt, dtype, B, H, G, D, held, seed=rows + waves + splits)
    options = dict(cap=20.0, window=T, slopes=[0.02 / (j + 1) for j in range(H * G)])
    assert launched_kernel(r, n) == (rows, waves, splits, False)
    took = launched_kernel(r, n, **options)
    assert took == (rows, waves, splits, True) or (rows, D) == (64, 128) and took[0] == 32 and took[3]
    new = [max(0, n - 1 - 5 * b) for b in range(B)]
    r.tree_attend(n, new, out=r.dt)
    r.tree_attend(n, new, **options)
    r.tree_attend(n, shape="forest")


@types
@pytest.mark.parametrize("B,H,G,n,T,splits", [(2, 1, 16, 128, 4600, 16), (4, 4, 8, 64, 4000, 8), (4, 8, 8, 64, 2500, 4),
                                              (8, 8, 8, 64, 2500, 2)])
def test_padded_chunks_in_splits(dtype, B, H, G, n, T, splits):
    """Chunks of cached tokens whose sequences take fewer than n, one none: the splits'
    parts of the other rows hold NaNs, their outputs are left as they were."""
    new = [n - 29] + [max(0, n // 2 - 13 * b) for b in range(1, B - 1)] + [0]
    held = [T + n - 29 * b for b in range(B)]
    r = Filled("e4m3", dtype, B, H, G, 64, held)
    past = [x - m for x, m in zip(held, new)]
    q = r.randn(B, H * G, n, 64).to(r.dt)
    for b, m in enumerate(new):
        q[b, :, m:] = math.nan
    o = torch.full(q.shape, 7.5, device="cuda")
    need = rq.rq_block_attention_workspace(r.c.desc, n, max(held))
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    dq, dp, dn = q.cuda(), ints(past), ints(new)
    torch.cuda.synchronize()

    def call(stream=None):
        rq.rq_block_attention(r.c.desc, 0, dp, dq, o, ws, new_len=dn, max_tokens=max(held), stream=stream)
    kernels = launches(call)
    assert "block_merge_rows_kernel" in kernels[1][0]
    assert kernels[0][1][0] == (n * G + 127) // 128 * B * H * splits
    call()
    whole, keys, values = r.u, np.zeros((B, H, n, 64)), np.zeros((B, H, n, 64))
    r.u = []
    for b, p in enumerate(past):
        r.u.append([Held(*(u.x[i][:p] for i in (0, 1)), u.pos[:p]) for u in whole[b]])
        for h, u in enumerate(whole[b]):
            keys[b, h, :new[b]], values[b, h, :new[b]] = (u.x[i][p:] for i in (0, 1))
    r.compare_tree(o, q, torch.from_numpy(keys).float(), torch.from_numpy(values).float(), new,
                   [np.tril(np.ones((m, m), bool)) for m in new], [list(range(m)) for m in new])


@pytest.mark.parametrize("n", [4, 40])
def test_trees_of_two_caches_at_once(n):
    """Two caches' calls in graphs on two streams, neither waited for before the other
    starts, with nodes for up to 16 rows and for more."""
    made = []
    for i in range(2):
        r = Filled(("int8", "e4m3")[i], "bf16", 2, 2, 4, 64, [3000, 2000 + 500 * i], seed=i)
        parents = [some_parents(n, 10 * i + b) for b in range(2)]
        q, (k, v) = r.randn(2, 8, n, 64).to(r.dt), r.nodes(n)
        layout = rq.DraftTree(ints(parents))
        d = [x.cuda() for x in (q, k, v)]
        o = torch.full(q.shape, 7.5, device="cuda")
        r.c.tree_attention(0, *d, layout, o)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(50):
                r.c.tree_attention(0, *d, layout, o)
        made.append((r, parents, q, k, v, o, stream, graph, layout, d))
    for _ in range(3):
        for r, parents, q, k, v, o, stream, graph, layout, d in made:
            with torch.cuda.stream(stream):
                o.fill_(7.5)
                graph.replay()
        torch.cuda.synchronize()
        for r, parents, q, k, v, o, stream, graph, layout, d in made:
            r.compare_tree(o, q, k, v, [n, n], [tree.sees(p) for p in parents],
                           [[len(c) - 1 for c in tree.ancestors(p)] for p in parents])


def test_the_oracle_s_rows_at_once():
    """attend_at_once against tree.attend."""
    g = np.random.default_rng(3)
    for L, window, cap, slopes in ((0, 0, 0.0, None), (9, 3, 4.0, [0.1, 0.0]), (40, 0, 0.0, [0.3, 0.2])):
        u = Held(g.standard_normal((L, 64)), g.standard_normal((L, 64)), np.cumsum(g.integers(1, 4, L)))
        p = some_parents(6, L)
        a = (u, g.standard_normal((6, 64)), g.standard_normal((6, 64)), tree.sees(p) & (g.random((6, 6)) < 0.7),
             [len(c) - 1 for c in tree.ancestors(p)], g.standard_normal((6, 2, 64)), 0.1, cap, window, slopes)
        np.testing.assert_allclose(attend_at_once(*a)[0], tree.attend(*a), rtol=0, atol=1e-13)
