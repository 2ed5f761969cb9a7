"""The block-scaled 8-bit cache on the GPU against its oracle: cache contents
bit for bit, attention and weights within bounds that follow from the
arithmetic.

Bounds.  With A a row's largest sum of |scale log2(e) q_c k_c|, a score (log2
units) is off by at most D 2^-24 A (fp32 sums of D exact products, any order)
plus D 2^-25 A' for bf16 queries held as fp16 (A' with |q_c| replaced by the
row's largest) plus four roundings of the score itself; a softmax ratio by
twice that times ln 2, plus the exponential's error (2^-22 each) and the sums'
(fp32, one rounding a term in each of at most T / 4 + 64 steps).  Values add
2^-21 of the largest one (22-bit products, scale)."""
import math

import numpy as np
import pytest
import torch

import paper_2605_06675_amd as rq
from oracle import block

pytestmark = pytest.mark.gpu
FMT = {"int8": (rq.RQ_INT8, block.INT8), "e4m3": (rq.RQ_E4M3, block.E4M3)}
DT = {"bf16": (rq.RQ_BF16, torch.bfloat16), "fp16": (rq.RQ_F16, torch.float16)}


def rounder(dt):
    return lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).float().numpy()


class Rig:
    """A device cache whose unused memory holds NaNs, and its oracle units."""

    def __init__(self, fmt="int8", dtype="bf16", B=2, H=2, G=2, D=128, cap=128, weights=True, seed=0,
                 layers=1, layer=0):
        self.fmt, self.B, self.H, self.G, self.D, self.cap = fmt, B, H, G, D, cap
        self.rdt, self.dt = DT[dtype]
        self.layer = layer
        self.g = torch.Generator().manual_seed(seed)
        self.c = rq.BlockCache(FMT[fmt][0], self.rdt, layers, B, H, H * G, D, cap, weights=weights)
        self.c.codes.fill_(0x7f)                      # e4m3: NaN
        self.c.scales.fill_(math.nan)
        self.c.tail.fill_(math.nan)
        self.c.positions.fill_(-(1 << 30))
        if weights:
            self.c.weights.fill_(math.nan)
        self.u = [[block.Unit(FMT[fmt][1], D, rounder(self.dt)) for _ in range(H)] for _ in range(B)]
        self.channel = torch.exp(torch.randn(H, 1, D, generator=self.g))

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g)

    def kv(self, n, new=None, size=1.0):
        k = self.randn(self.B, self.H, n, self.D) * self.channel * size
        k = k.clamp(-65504, 65504).to(self.dt)        # (keys must be finite in fp16)
        v = (self.randn(self.B, self.H, n, self.D) * size).to(self.dt)
        if new is not None:                           # padding rows hold NaNs
            for b, m in enumerate(new):
                k[b, :, m:], v[b, :, m:] = math.nan, math.nan
        return k, v

    def append(self, n, new=None, size=1.0, kv=None):
        k, v = self.kv(n, new, size) if kv is None else kv
        self.c.append(self.layer, k.cuda(), v.cuda(), None if new is None else ints(new))
        self.took(k, v, new)

    def took(self, k, v, new=None):
        for b in range(self.B):
            m = k.shape[2] if new is None else new[b]
            for h in range(self.H):
                self.u[b][h].append(k[b, h, :m].float().numpy(), v[b, h, :m].float().numpy())

    def lengths(self):
        return [self.u[b][0].length for b in range(self.B)]

    def check(self, weights=True):
        """Buffers equal the oracle's; what it does not hold is untouched."""
        c, L = self.c, self.layer
        sh = (c.desc.n_layers, self.B, self.H)
        codes = c.codes.cpu().numpy().reshape(*sh, 2, self.cap, self.D)[L]
        scales = c.scales.cpu().numpy().reshape(*sh, 2, self.cap // 32)[L]
        tail = c.tail.cpu().float().numpy().reshape(*sh, 2, 32, self.D)[L]
        pos = c.positions.cpu().numpy().reshape(*sh, self.cap)[L]
        assert c.lengths[L].tolist() == self.lengths()
        for b in range(self.B):
            for h in range(self.H):
                u = self.u[b][h]
                n, full = u.length, u.length // 32 * 32
                for s in (0, 1):
                    np.testing.assert_array_equal(codes[b, h, s, :full], u.codes[s])
                    np.testing.assert_array_equal(scales[b, h, s, :full // 32], u.scales[s])
                    np.testing.assert_array_equal(tail[b, h, s, :n - full], u.tail[s])
                    assert (codes[b, h, s, full:] == 0x7f).all()
                    assert np.isnan(scales[b, h, s, full // 32:]).all()
                np.testing.assert_array_equal(pos[b, h, :n], u.pos)
                assert (pos[b, h, n:] == -(1 << 30)).all()

    def weights(self):
        return self.c.weights.cpu().view(-1, self.B, self.H, self.cap)[self.layer].double().numpy()

    def bounds(self, b, h, q, scale, cap, slopes):
        """(bound on a softmax ratio, largest |value|) for each row of q
        [n][G][D]."""
        u = self.u[b][h]
        K, V = (u.values(s).astype(np.float64) for s in (0, 1))
        q, scale = np.abs(q.astype(np.float64)), abs(scale)
        a = scale * 1.4427 * (q @ np.abs(K).T).max(-1)
        a2 = scale * 1.4427 * (q.max(-1) * np.abs(K).sum(-1).max())
        far = 0.0 if slopes is None else 1.4427 * float(np.max(slopes)) * float(u.pos.max())
        s = self.D * 2.0 ** -24 * a + (self.D * 2.0 ** -25 * a2 if self.dt == torch.bfloat16 else 0)
        # a capped score never errs by more than the uncapped one, and by the tanh's own 2^-21
        s = s + 4 * 2.0 ** -24 * (a + far) + (1.4427 * cap * 2.0 ** -21 if cap else 0)
        ratio = 2 * s * math.log(2) + 2.0 ** -21 + (u.length / 4 + 64) * 2.0 ** -24
        return ratio, (np.abs(V).max() if len(V) else 0.0)

    def attend(self, n, new=None, out=torch.float32, scale=None, cap=0.0, window=0, slopes=None,
               accumulate=False, q=None, size=1.0, stream=None, max_tokens=None):
        """One call, checked against the oracle."""
        q = (self.randn(self.B, self.H * self.G, n, self.D) * size).to(self.dt) if q is None else q
        if new is not None:
            for b, m in enumerate(new):
                q[b, :, m:] = math.nan
        past = [L - (n if new is None else new[b]) for b, L in enumerate(self.lengths())]
        bound = max(self.lengths() + [n]) if max_tokens is None else max_tokens
        before = self.weights() if accumulate else None
        o = torch.full(q.shape, 7.5, dtype=out, device="cuda")
        ws = torch.full((max(16, rq.rq_block_attention_workspace(self.c.desc, n, bound, accumulate, window)),),
                        0xff, dtype=torch.uint8, device="cuda")
        rq.rq_block_attention(self.c.desc, self.layer, ints(past), q.cuda(), o, ws,
                              None if new is None else ints(new), bound, scale, cap, window,
                              None if slopes is None else torch.tensor(slopes).cuda(), accumulate, stream)
        torch.cuda.synchronize()
        self.compare(q, o, new, scale, cap, window, slopes, accumulate, before)
        return o

    def compare(self, q, o, new=None, scale=None, cap=0.0, window=0, slopes=None, accumulate=False,
                before=None):
        n, G, out = q.shape[2], self.G, o.dtype
        scale = self.D ** -0.5 if scale is None else scale
        half = 0.0 if out == torch.float32 else torch.finfo(out).eps / 2
        after = self.weights() if accumulate else None
        o = o.cpu().double().numpy()
        for b in range(self.B):
            m = n if new is None else new[b]
            assert (o[b, :, m:] == 7.5).all()
            for h in range(self.H):
                if m == 0:
                    continue
                u = self.u[b][h]
                qq = q[b, h * G:(h + 1) * G, :m].float().numpy().transpose(1, 0, 2)
                sl = None if slopes is None else np.asarray(slopes[h * G:(h + 1) * G])
                old = u.weight.copy()
                want = u.attend(qq, scale, cap, window, sl, accumulate)
                ratio, big = self.bounds(b, h, qq, scale, cap, sl)
                got = o[b, h * G:(h + 1) * G, :m].transpose(1, 0, 2)
                err = np.abs(got - want)
                tol = (ratio[..., None] + 2.0 ** -21) * big + half * np.abs(want) + 1e-30
                if out == torch.float16:
                    tol = tol + 2.0 ** -25
                assert (err <= tol).all(), (b, h, float((err / tol).max()))
                if accumulate:
                    L = u.length
                    add = u.weight - old
                    grown = after[b, h, :L] - before[b, h, :L]
                    tol = ratio.max() * add + 2.0 ** -24 * (np.abs(after[b, h, :L]) + m * G * add)
                    worst = np.abs(grown - add) / (tol + 1e-30)
                    at = int(worst.argmax())
                    assert worst[at] <= 1, (b, h, at, float(worst[at]), float(grown[at]), float(add[at]))
                    assert np.isnan(after[b, h, L:]).all()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


both = pytest.mark.parametrize("fmt", ["int8", "e4m3"])
types = pytest.mark.parametrize("dtype", ["bf16", "fp16"])


# ------------------------------------------------------------------- append
@both
@types
@pytest.mark.parametrize("D", [64, 128])
def test_append_in_pieces(fmt, dtype, D):
    r = Rig(fmt, dtype, D=D, cap=192)
    for n in (1, 30, 1, 1, 31, 64, 33, 3):
        r.append(n)
        r.check()
    assert (r.weights()[:, :, :164] == 0).all() and np.isnan(r.weights()[:, :, 164:]).all()


@both
def test_append_ragged_and_padded(fmt):
    r = Rig(fmt, "fp16", B=4, D=64, cap=160)
    for n, new in ((50, [50, 0, 1, 32]), (64, [14, 64, 0, 33]), (9, [9, 0, 1, 2])):
        r.append(n, new)
        r.check()


@both
@types
def test_append_sizes(fmt, dtype):
    """Zeros, one spike, the dtype's largest and smallest numbers, ties."""
    r = Rig(fmt, dtype, B=1, H=1, cap=192)
    n, big = 32, float(torch.finfo(r.dt).max) if dtype == "fp16" else 2.0 ** 55
    z = torch.zeros(1, 1, n, 128, dtype=r.dt)
    spike, most, small = z.clone(), z.clone(), z.clone()
    spike[0, 0, 17, 5] = -3.0
    most[0, 0] = torch.where(torch.rand(n, 128, generator=r.g) < 0.5, big, -big).to(r.dt)
    small[0, 0] = (r.randn(n, 128) * float(torch.finfo(r.dt).smallest_normal)).to(r.dt)
    ties = (torch.arange(n * 128).view(1, 1, n, 128) % 255 - 127).to(r.dt) / 2
    for x in (z, spike, most, small, ties):
        r.append(n, kv=(x, -x))
    r.check()


@pytest.mark.parametrize("D", [64, 128])
def test_append_strided_and_unaligned_rows(D):
    r = Rig("int8", "bf16", B=2, H=3, D=D, cap=128)
    n = 45
    k, v = r.kv(n)
    dk = torch.empty(2, n, 3, D, dtype=r.dt, device="cuda").transpose(1, 2)     # [B][n][H][D]
    dk.copy_(k)
    flat = torch.empty(2 * 3 * n * (D + 3) + 1, dtype=r.dt, device="cuda")
    dv = flat[1:].view(2, 3, n, D + 3)[..., 2:D + 2]                            # any element
    dv.copy_(v)
    r.c.append(0, dk, dv)
    r.took(k, v)
    r.check()
    k1, v1 = r.kv(1)                       # one token broadcast over the batch
    k1[1], v1[1] = k1[0], v1[0]
    r.c.append(0, k1[:1].cuda().expand(2, -1, -1, -1), v1[:1].cuda().expand(2, -1, -1, -1))
    r.took(k1, v1)
    r.check()


def test_append_stops_at_the_capacity():
    r = Rig("int8", B=3, H=1, cap=64)
    r.append(40, [40, 20, 40])
    k, v = r.kv(40)
    rq.rq_block_append(r.c.desc, 0, ints([40, 20, -5]), k.cuda(), v.cuda())
    r.c.lengths[0] = ints([64, 60, 40])
    u = r.u
    u[0][0].append(k[0, 0, :24].float().numpy(), v[0, 0, :24].float().numpy())
    u[1][0].append(k[1, 0].float().numpy(), v[1, 0].float().numpy())
    u[2][0] = block.Unit(block.INT8, 128, rounder(r.dt))     # -5 counts as 0
    u[2][0].append(k[2, 0].float().numpy(), v[2, 0].float().numpy())
    r.check()
    rq.rq_block_append(r.c.desc, 0, ints([64, 64, 1000]), k.cuda(), v.cuda(), ints([3, 0, -1]))
    r.c.lengths[0] = ints([64, 60, 40])
    r.check()


def test_layers_are_apart():
    r = Rig("e4m3", layers=3, layer=1, cap=64)
    r.append(40)
    r.check()
    c = r.c.codes.view(3, -1)
    assert (c[0] == 0x7f).all() and (c[2] == 0x7f).all()
    assert torch.isnan(r.c.tail.view(3, -1)[[0, 2]]).all()
    r.attend(3, accumulate=True)
    assert torch.isnan(r.c.weights.view(3, -1)[[0, 2]]).all()


# ---------------------------------------------------------------- attention
@both
@types
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [1, 31, 32, 33, 100, 1000])
def test_attend_one_token(fmt, dtype, D, L):
    r = Rig(fmt, dtype, G=4, D=D, cap=1024)
    r.append(L)
    r.attend(1)


@pytest.mark.parametrize("G", [1, 3, 6, 16])
@pytest.mark.parametrize("n", [2, 5, 40])
def test_attend_several_tokens(G, n):
    r = Rig("e4m3", "bf16", H=1, G=G, D=64, cap=256)
    r.append(170)
    r.attend(n)
    r.append(n)
    r.attend(n, out=torch.bfloat16)


@both
@types
@pytest.mark.parametrize("n", [1, 7, 130])
@pytest.mark.parametrize("kw", [dict(cap=20.0), dict(window=1), dict(window=50), dict(window=4000),
                                dict(slopes=[0.5, 0.25, 0.0, 1.0]),
                                dict(cap=5.0, window=33, slopes=[0.01, 0.02, 0.03, 0.04])])
def test_attend_masks_and_biases(fmt, dtype, n, kw):
    r = Rig(fmt, dtype, D=64, cap=512)
    r.append(333)
    r.attend(n, accumulate=True, **kw)


@both
def test_attend_ragged(fmt):
    """Empty sequences, padded rows of NaNs, lengths inside one block."""
    r = Rig(fmt, "bf16", B=5, G=3, cap=256)
    r.append(200, [200, 0, 5, 64, 33])
    new = [9, 0, 1, 4, 9]
    r.append(9, new)
    r.attend(9, new, accumulate=True)
    r.attend(9, new, out=torch.float16, window=3, max_tokens=256)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", [1e-4, 1.0, 2000.0])
def test_attend_value_and_query_sizes(dtype, size):
    r = Rig("int8", dtype, cap=256)
    r.append(64, size=size)
    r.append(32, size=size * 0.01)
    r.append(32)
    r.append(9, size=size)
    r.attend(1, scale=0.05 / size ** 2 if size > 1 else None, size=size)
    r.attend(6, scale=0.05 / size ** 2 if size > 1 else None, size=size)


@both
def test_attend_equal_scores_give_the_mean(fmt):
    """Queries of zero: every probability is the same, so the output shows
    the products' 22 bits and the sums alone."""
    r = Rig(fmt, "bf16", cap=2048)
    r.append(1500)
    q = torch.zeros(2, 4, 1, 128, dtype=r.dt)
    o = r.attend(1, q=q).cpu().double().numpy()
    for b in range(2):
        for h in range(2):
            mean = r.u[b][h].values(1).astype(np.float64).mean(0)
            assert np.abs(o[b, 2 * h, 0] - mean).max() <= 4 * 2.0 ** -22 * np.abs(r.u[b][h].values(1)).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kw", [dict(), dict(cap=7.0), dict(slopes=[0.1, 0.2, 0.3, 0.4])])
@pytest.mark.parametrize("n", [1, 6, 70])
def test_attend_negative_and_zero_scale(dtype, kw, n):
    r = Rig("int8", dtype, D=64, cap=256)
    r.append(201)
    for scale in (-0.2, 0.0):
        r.attend(n, scale=scale, accumulate=True, **kw)


@both
@pytest.mark.parametrize("dtype,size", [("fp16", 2.0 ** -10), ("bf16", 2.0 ** -60), ("fp16", 2.0 ** 12),
                                        ("bf16", 2.0 ** 40)])
@pytest.mark.parametrize("zeros", [0, 32, 64])
@pytest.mark.parametrize("L", [7, 64, 100])
@pytest.mark.parametrize("n", [1, 40])
def test_attend_precision_of_small_and_large_values(fmt, dtype, size, zeros, L, n):
    """Queries of zero: the output is the values' mean, to 22 bits of their
    largest, wherever their magnitude lies, behind blocks of zeros, in the
    tail, and to 2^-25 in each of its 32 numbers' fp16 forms."""
    r = Rig(fmt, dtype, cap=256)
    if zeros:
        z = torch.zeros(2, 2, zeros, 128, dtype=r.dt)
        r.append(zeros, kv=(z, z))
    k, v = r.kv(max(L, n))
    r.append(max(L, n), kv=(k, (v.float() * size).to(r.dt)))
    o = r.attend(n, q=torch.zeros(2, 4, n, 128, dtype=r.dt)).cpu().double().numpy()
    for b in range(2):
        for h in range(2):
            V = r.u[b][h].values(1).astype(np.float64)
            mean = V[:len(V) - n + 1].mean(0)
            assert np.abs(o[b, 2 * h, 0] - mean).max() <= 6 * 2.0 ** -22 * np.abs(V).max()


def test_attend_zero_blocks():
    r = Rig("e4m3", "fp16", cap=128)
    z = torch.zeros(2, 2, 32, 128, dtype=r.dt)
    r.append(32, kv=(z, z))
    r.attend(2)
    r.append(40)
    r.append(32, kv=(z, z))
    r.attend(2)


def test_attend_one_dominant_score_far_back():
    """A late maximum rescales what came before, an early one never moves."""
    for at in (3, 700):
        r = Rig("int8", "bf16", B=1, H=1, G=1, cap=1024)
        k, v = r.kv(800)
        q = r.randn(1, 1, 1, 128).to(r.dt)
        k[0, 0, at] = (q[0, 0, 0].float() * 4).to(r.dt)
        r.append(800, kv=(k, v))
        r.attend(1, q=q)


def test_attend_strided_unaligned_and_long_batch():
    r = Rig("e4m3", "bf16", B=2, H=2, G=2, D=64, cap=96)
    r.append(77)
    n, q = 4, r.randn(2, 4, 4, 64).to(r.dt)
    dq = torch.empty(2 * n * 4 * 67 + 1, dtype=r.dt, device="cuda")[1:].view(2, n, 4, 67)[..., 1:65].transpose(1, 2)
    dq.copy_(q)
    for out in (torch.float32, torch.bfloat16):
        do = torch.full((2 * n * 4 * 67 + 1,), 7.5, dtype=out, device="cuda")[1:].view(2, n, 4, 67)
        o = do[..., 2:66].transpose(1, 2)
        ws = torch.empty(rq.rq_block_attention_workspace(r.c.desc, n, 77) + 16, dtype=torch.uint8, device="cuda")
        rq.rq_block_attention(r.c.desc, 0, ints([73, 73]), dq, o, ws, max_tokens=77)
        r.compare(q, o)
        assert (do[..., :2] == 7.5).all() and (do[..., 66:] == 7.5).all()


def test_lengths_out_of_range_are_taken_as_the_nearest():
    r = Rig("int8", "bf16", B=2, cap=96)
    r.append(96, [96, 2])
    q = r.randn(2, 4, 2, 128).to(r.dt).cuda()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def call(past, new):
        o = torch.full(q.shape, 7.5, device="cuda")
        rq.rq_block_attention(r.c.desc, 0, ints(past), q, o, ws, ints(new))
        return o
    torch.testing.assert_close(call([1000, -3], [2, 2]), call([94, 0], [2, 2]), rtol=0, atol=0)
    torch.testing.assert_close(call([94, 50], [9, -1]), call([94, 50], [2, 0]), rtol=0, atol=0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,G,L", [(1, 1, 1, 500), (1, 1, 1, 4000), (1, 1, 2, 9000), (1, 2, 3, 2000),
                                     (2, 4, 8, 1500), (1, 8, 4, 4000), (1, 4, 16, 1100), (3, 5, 4, 3001)])
def test_attend_split_sequences(D, B, H, G, L):
    """Splits merged by the last workgroup and by a launch of their own."""
    r = Rig("int8", "bf16", B=B, H=H, G=G, D=D, cap=(L + 63) // 32 * 32)
    k, v = r.kv(L)
    r.c.append(0, k.cuda(), v.cuda())
    for b in range(B):
        for h in range(H):
            u, full = r.u[b][h], L // 32 * 32
            for s, x in ((0, k), (1, v)):
                part = [block.quantize(block.INT8, x[b, h, i:i + 32].float().numpy()) for i in range(0, full, 32)]
                u.codes[s] = np.concatenate([c for c, _ in part])
                u.scales[s] = np.array([y for _, y in part], np.float32)
                u.tail[s] = x[b, h, full:].float().numpy()
            u.pos, u.weight = np.arange(L), np.zeros(L)
    r.attend(1)
    q = r.randn(B, H * G, 1, D).to(r.dt)
    first = r.attend(1, q=q)
    r.c.desc.counters, counters = None, r.c.desc.counters
    other = r.attend(1, q=q)
    r.c.desc.counters = counters
    torch.testing.assert_close(first, other, rtol=1e-5, atol=1e-6)
    assert (r.c.desc._buffers[-1] == 0).all()


def test_attend_repeats_bit_for_bit():
    r = Rig("int8", "bf16", B=1, cap=4096)
    r.append(4001)
    q = r.randn(1, 4, 1, 128).to(r.dt)
    a, w = r.attend(1, q=q), r.c.weights.clone()
    assert torch.equal(a, r.attend(1, q=q))
    r.attend(1, q=q, accumulate=True)
    w1 = r.c.weights.clone()
    r.c.weights.copy_(w)
    for u in r.u[0]:
        u.weight[:] = 0
    r.attend(1, q=q, accumulate=True)
    assert torch.equal(w1[~torch.isnan(w1)], r.c.weights[~torch.isnan(w1)])


def between_roundings(o, want, tol):
    """Every output is a rounding of some number within tol of want."""
    lo, hi = (torch.from_numpy(x).to(o.dtype).double() for x in (want - tol, want + tol))
    o = o.cpu().double()
    return bool(((lo <= o) & (o <= hi)).all())


@both
@types
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_probabilities_hold_22_bits(fmt, dtype, D):
    """Queries of zero: a 16-bit output is the values' mean, rounded once, with
    as little before that as fp32 outputs show."""
    r = Rig(fmt, dtype, D=D, cap=160)
    r.append(150)
    n, q = 40, torch.zeros(2, 4, 40, D, dtype=r.dt)
    o = r.attend(n, q=q, out=r.dt).cpu()
    for b in range(2):
        for h in range(2):
            V = r.u[b][h].values(1).astype(np.float64)
            want = np.stack([V[:150 - n + 1 + i].mean(0) for i in range(n)])
            tol = 6 * 2.0 ** -22 * np.abs(V).max()
            for g in range(2):
                assert between_roundings(o[b, 2 * h + g], want, tol), (b, h)


@pytest.mark.parametrize("cap", [20.0, 300.0, 1e4, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("n,dtype,out", [(1, "bf16", "fp32"), (40, "bf16", "bf16"), (40, "bf16", "fp32"),
                                         (70, "fp16", "fp16")])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_large_caps(cap, n, dtype, out, D):
    """A capped score errs relative to itself, not to the cap: where the cap is
    far above the scores, the result is that of none."""
    r = Rig("e4m3", dtype, D=D, cap=192)
    r.append(130)
    q = (r.randn(2, 4, n, D) * 2).to(r.dt)
    before = r.weights()
    o = r.attend(n, q=q, cap=cap, accumulate=True, out={**DT, "fp32": (0, torch.float32)}[out][1])
    after, o, scale = r.weights(), o.cpu(), D ** -0.5
    for b in range(2):
        for h in range(2):
            u = block.Unit(r.u[b][h].fmt, D, None)
            u.__dict__.update({**r.u[b][h].__dict__, "weight": np.zeros(130)})
            qq = q[b, 2 * h:2 * h + 2].float().numpy().transpose(1, 0, 2)
            want = u.attend(qq, scale, cap, accumulate=True)
            ratio, big = r.bounds(b, h, qq, scale, 0.0, None)
            # tanh to 2^-21 of itself, the score not above the row's sum of |q k|
            K = np.abs(u.values(0).astype(np.float64))
            ratio = ratio + 2 * 2.0 ** -21 * scale * (np.abs(qq.astype(np.float64)) @ K.T).max(-1)
            got = o[b, 2 * h:2 * h + 2].transpose(0, 1)
            assert between_roundings(got, want, (ratio[..., None] + 2.0 ** -21) * big), (b, h)
            add = after[b, h, :130] - before[b, h, :130]
            tol = ratio.max() * u.weight + 2.0 ** -24 * (after[b, h, :130] + 2 * n * u.weight)
            assert (np.abs(add - u.weight) <= tol + 1e-30).all(), (b, h)


@both
@pytest.mark.parametrize("n,G", [(1, 1), (5, 2), (30, 2), (40, 4)])
@pytest.mark.parametrize("window", [0, 1])
def test_attend_scores_far_below_zero(fmt, n, G, window):
    """Scores of -1.4e31, alike for all tokens a row sees: of the unfinished
    block its mean, behind a window of one the token itself."""
    if not window and n > 31:
        n = 31
    r = Rig(fmt, "bf16", G=G, cap=64)
    k, v = r.kv(n)
    k[:] = 2.0 ** 50
    r.append(n, kv=(k, v))
    o = torch.full((2, 2 * G, n, 128), 7.5, device="cuda")
    ws = torch.empty(rq.rq_block_attention_workspace(r.c.desc, n, 64, True), dtype=torch.uint8, device="cuda")
    q = torch.full((2, 2 * G, n, 128), -2.0 ** 50, dtype=r.dt, device="cuda")
    rq.rq_block_attention(r.c.desc, 0, ints([0, 0]), q, o, ws, max_tokens=64, window=window, accumulate=True)
    o, w = o.cpu().double().numpy(), r.weights()
    for b in range(2):
        for h in range(2):
            V = r.u[b][h].values(1).astype(np.float64)
            seen = [V[i:i + 1] if window else V[:i + 1] for i in range(n)]
            want = np.stack([x.mean(0) for x in seen])
            for g in range(G):
                assert np.abs(o[b, h * G + g] - want).max() <= 8 * 2.0 ** -22 * np.abs(V).max()
            add = G * (np.ones(n) if window else np.cumsum(1 / np.arange(n, 0, -1.0))[::-1])
            np.testing.assert_allclose(w[b, h, :n], add, rtol=1e-5)


@pytest.mark.parametrize("fmt,most", [("int8", 127.0), ("e4m3", 448.0)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_attend_equal_scores_of_any_size(fmt, most, sign, n):
    """Keys alike, whose codes and scale are exact, and scores of 2^33 and more:
    still the mean of values whose blocks' scales differ."""
    r = Rig(fmt, "bf16", cap=256)
    for size in (1.0, 100.0, 0.01, 1.0):
        k, v = r.kv(50)
        k[:] = most * 2.0 ** 10
        r.append(50, kv=(k, (v * size).to(r.dt)))
    q = torch.full((2, 4, n, 128), sign * 2.0 ** 10, dtype=r.dt)
    o = r.attend(n, q=q, scale=1.0, accumulate=True).cpu().double().numpy()
    for b in range(2):
        for h in range(2):
            V = r.u[b][h].values(1).astype(np.float64)
            want = np.stack([V[:201 - n + i].mean(0) for i in range(n)])
            for g in range(2):
                assert np.abs(o[b, 2 * h + g] - want).max() <= 6 * 2.0 ** -22 * np.abs(V).max()
            np.testing.assert_allclose(r.weights()[b, h, :200 - n], 2 * sum(1 / (201 - n + i) for i in range(n)),
                                       rtol=1e-5)


@both
@pytest.mark.parametrize("dtype,size,scale", [("bf16", 2.0 ** 17, 1.0), ("bf16", 2.0 ** 17, -1.0),
                                              ("fp16", 2.0 ** 5, 2.0 ** 20)])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_attend_large_scores_pick_one_token(fmt, dtype, size, scale, n):
    """Scores of 2^32 and more: the values of the largest, wherever it leads by
    more than the products' rounding."""
    r = Rig(fmt, dtype, cap=256)
    k, v = r.kv(200)
    r.append(200, kv=((k.float() * size).to(r.dt), v))
    q = (r.randn(2, 4, n, 128) * size).to(r.dt)
    o = r.attend(n, q=q, scale=scale, accumulate=True).cpu().double().numpy()
    sure = 0
    for b in range(2):
        for h in range(2):
            K, V = (r.u[b][h].values(s).astype(np.float64) for s in (0, 1))
            for g in range(2):
                for i in range(n):
                    qq = q[b, 2 * h + g, i].double().numpy()
                    seen = K[:201 - n + i]
                    x, err = scale * (seen @ qq), np.abs(scale) * (np.abs(seen) @ np.abs(qq)).max() * 2.0 ** -16
                    top = np.argsort(x)[-2:]
                    if x[top[1]] - x[top[0]] > err + 100:
                        sure += 1
                        assert np.abs(o[b, 2 * h + g, i] - V[top[1]]).max() <= 2.0 ** -20 * np.abs(V).max()
    assert sure >= 4 * n


@pytest.mark.parametrize("n,L", [(1, 90), (1, 1900), (5, 1900), (40, 300)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30])
def test_attend_windows_beyond_every_position(n, L, window):
    """No limit, written as a window: results and weights of none."""
    r = Rig("int8", "bf16", G=2, D=64, cap=2048)
    r.append(L)
    r.attend(n, window=window, accumulate=True)
    r.attend(n, window=window, max_tokens=2048, accumulate=True)


def fill(r, L):
    """Appends L tokens to every sequence; the oracle's blocks at once."""
    k, v = r.kv(L)
    r.c.append(r.layer, k.cuda(), v.cuda())
    full = L // 32 * 32
    for b in range(r.B):
        for h in range(r.H):
            u = r.u[b][h]
            for s, x in ((0, k), (1, v)):
                part = [block.quantize(u.fmt, x[b, h, i:i + 32].float().numpy()) for i in range(0, full, 32)]
                u.codes[s] = np.concatenate([c for c, _ in part])
                u.scales[s] = np.array([y for _, y in part], np.float32)
                u.tail[s] = x[b, h, full:].float().numpy()
            u.pos, u.weight = np.arange(L), np.zeros(L)


OPTIONS = [dict(), dict(cap=15.0), dict(window=70), dict(slopes=True), dict(cap=9.0, window=150, slopes=True)]


@both
@pytest.mark.parametrize("B,H,G,n,L", [(1, 8, 2, 100, 301), (2, 8, 4, 33, 160), (4, 4, 3, 90, 90), (3, 1, 8, 70, 500)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("kw", OPTIONS)
def test_prompt_units_and_options(fmt, B, H, G, n, L, dtype, out, kw):
    """Prompts of 8 and 16 units and others, several tiles of rows, split and
    not, 128 channels: outputs of every type, masks and biases, weights."""
    r = Rig(fmt, dtype, B=B, H=H, G=G, D=128, cap=512)
    fill(r, L)
    if "slopes" in kw:
        kw = {**kw, "slopes": (2.0 ** (-8.0 * np.arange(1, H * G + 1) / (H * G))).astype(np.float32).tolist()}
    r.attend(n, accumulate=True, out={**DT, "fp32": (0, torch.float32)}[out][1], **kw)


@pytest.mark.parametrize("dtype,n,G,L", [("fp16", 512, 16, 4609), ("bf16", 520, 8, 4192), ("fp16", 256, 16, 8100)])
def test_long_chunks_split_in_two(dtype, n, G, L):
    """Chunks of many rows behind many tokens, uneven ones, against an fp64
    product on the device."""
    B, H, D, cap = 2, 4 if G == 16 else 8, 64, (L + 31) // 32 * 32
    r = Rig("int8", dtype, B=B, H=H, G=G, D=D, cap=cap)
    lengths, new = [L, L - 700], [n, n - 90]
    k, v = (x.cuda() for x in r.kv(L, lengths))
    r.c.append(0, k, v, ints(lengths))
    q = r.randn(B, H * G, n, D).to(r.dt).cuda()
    q[1, :, n - 90:] = math.nan
    o = r.c.attention(0, q, torch.full(q.shape, 7.5, device="cuda"), ints(new), accumulate=True)
    codes = r.c.codes.view(torch.int8).view(B, H, 2, cap, D)
    scales, tail = r.c.scales.view(B, H, 2, cap // 32), r.c.tail.view(B, H, 2, 32, D)
    for b in range(B):
        T, m = lengths[b], new[b]
        full = T // 32 * 32
        assert (o[b, :, m:] == 7.5).all()
        hide = torch.arange(T, device="cuda") > torch.arange(T - m, T, device="cuda")[:, None]
        for h in range(H):
            K, V = (torch.cat([(codes[b, h, s, :full].float() * scales[b, h, s, :full // 32]
                                .repeat_interleave(32)[:, None]).double(), tail[b, h, s, :T - full].double()])
                    for s in (0, 1))
            add = torch.zeros(T, dtype=torch.float64, device="cuda")
            worst, big = 0.0, float(V.abs().max())
            for g in range(G):
                x = q[b, h * G + g, :m].double()
                p = torch.softmax((x @ K.T.contiguous() / math.sqrt(D)).masked_fill(hide, -math.inf), -1)
                add += p.sum(0)
                a = 1.4427 / math.sqrt(D) * (x.abs() @ K.abs().T.contiguous()).amax(-1)
                s = (D + 4) * 2.0 ** -24 * a
                if dtype == "bf16":
                    s += D * 2.0 ** -25 * 1.4427 / math.sqrt(D) * x.abs().amax(-1) * K.abs().sum(-1).max()
                ratio = 2 * s * math.log(2) + 2.0 ** -21 + (T / 4 + 64) * 2.0 ** -24
                worst = max(worst, float(ratio.max()))
                assert ((o[b, h * G + g, :m].double() - p @ V).abs() <= (ratio[:, None] + 2.0 ** -21) * big).all()
            w = r.c.weights.view(B, H, cap)[b, h, :T].double()
            assert ((w - add).abs() <= worst * add + 2.0 ** -24 * (1 + m * G) * add + 1e-30).all()


# ----------------------------------------------------------------- eviction
def evict(r, keep, sink, recent, weight=None):
    """Evicts r's cache; returns a rig around the new one, checked."""
    if weight is not None:
        w = torch.full((r.B, r.H, r.cap), math.nan)
        for b in range(r.B):
            for h in range(r.H):
                w[b, h, :r.u[b][h].length] = weight[b, h, :r.u[b][h].length]
        r.c.weights.view(r.B, r.H, r.cap).copy_(w)
    dev_w = r.weights()
    before = [t.clone() for t in (r.c.codes, r.c.scales, r.c.tail, r.c.positions, r.c.weights)]
    to = Rig(r.fmt, "bf16" if r.dt == torch.bfloat16 else "fp16", r.B, r.H, r.G, r.D,
             (keep + 31) // 32 * 32 + 32)
    r.c.evict(keep, sink, recent, into=to.c)
    for t, old in zip((r.c.codes, r.c.scales, r.c.tail, r.c.positions, r.c.weights), before):
        assert torch.equal(t.view(torch.uint8), old.view(torch.uint8))
    for b in range(r.B):
        for h in range(r.H):
            to.u[b][h] = r.u[b][h].evict(keep, sink, recent, dev_w[b, h, :r.u[b][h].length])
    to.channel = r.channel
    to.check()
    got = to.weights()
    for b in range(r.B):
        for h in range(r.H):
            n = to.u[b][h].length
            np.testing.assert_array_equal(got[b, h, :n], to.u[b][h].weight)
            assert np.isnan(got[b, h, n:]).all()
    return to


@both
@types
@pytest.mark.parametrize("D", [64, 128])
def test_evict_random_weights(fmt, dtype, D):
    r = Rig(fmt, dtype, B=3, D=D, cap=512)
    r.append(500, [500, 37, 200])
    to = evict(r, 131, 4, 20, torch.rand(3, 2, 512, generator=r.g))
    to.append(5)
    to.check()
    to.attend(5, window=90)


@pytest.mark.parametrize("kind", ["zero", "equal", "few", "levels", "tiny", "inf"])
def test_evict_ties_and_sizes(kind):
    r = Rig("int8", "bf16", B=1, H=2, D=64, cap=2112)
    r.append(2100)
    w = torch.rand(1, 2, 2112, generator=r.g)
    w = {"zero": w * 0, "equal": w * 0 + 0.37, "few": (w < 0.01).float(), "levels": (w * 7).floor(),
         "tiny": w * 1e-40, "inf": torch.where(w < 0.1, math.inf, w)}[kind]
    evict(r, 700, 3, 50, w)


@pytest.mark.parametrize("keep,sink,recent", [(1, 0, 1), (32, 31, 1), (33, 0, 33), (64, 4, 8), (99, 10, 20),
                                              (100, 0, 1), (101, 0, 1), (120, 50, 70)])
def test_evict_counts(keep, sink, recent):
    r = Rig("e4m3", "bf16", B=2, H=1, D=64, cap=128)
    r.append(100, [100, 0])
    evict(r, keep, sink, recent, torch.rand(2, 1, 128, generator=r.g))


@pytest.mark.parametrize("kind", ["random", "zero", "few", "late"])
def test_evict_long(kind):
    """A unit selected in several parts; ties across them."""
    r = Rig("int8", "fp16", B=1, H=1, D=64, cap=40032)
    k, v = r.kv(40001)
    r.c.append(0, k.cuda(), v.cuda())
    u = r.u[0][0]
    full = 40000
    q = [block.quantize(block.INT8, x[0, 0, i:i + 32].float().numpy()) for x in (k, v) for i in range(0, full, 32)]
    half = len(q) // 2
    for s in (0, 1):
        part = q[s * half:(s + 1) * half]
        u.codes[s] = np.concatenate([c for c, _ in part])
        u.scales[s] = np.array([x for _, x in part], np.float32)
        u.tail[s] = (k, v)[s][0, 0, full:].float().numpy()
    u.pos, u.weight = np.arange(40001), np.zeros(40001)
    r.check()
    w = -torch.log(torch.rand(1, 1, 40032, generator=r.g))
    w = {"random": w, "zero": w * 0, "few": (w < 0.01).float(), "late": (torch.arange(40032) > 37000).float()[None, None]}[kind]
    evict(r, 5000, 4, 64, w)


@pytest.mark.parametrize("L,cap", [(4000, 4096), (9001, 9024), (20001, 20032), (32768, 32768)])
@pytest.mark.parametrize("kind", ["random", "zero", "few"])
def test_evict_selection(L, cap, kind):
    """The kept slots alone, for units selected by one workgroup."""
    r = Rig("int8", "bf16", B=2, H=1, D=64, cap=cap)
    k, v = r.kv(L)
    r.c.append(0, k.cuda(), v.cuda())
    w = torch.rand(2, 1, cap, generator=r.g)
    w = {"random": w, "zero": w * 0, "few": (w < 0.01).float()}[kind]
    r.c.weights.view(2, 1, cap).copy_(w)
    keep = L // 3
    pos = r.c.evict(keep, 4, 30).positions.view(2, -1).cpu()
    for b in range(2):
        order = w[b, 0, :L].double()
        order[:4] = order[L - 30:] = 9.0
        rank = torch.sort(order, stable=True, descending=True)[1][:keep]
        assert torch.equal(pos[b, :keep].long(), torch.sort(rank)[0])


@pytest.mark.parametrize("L,cap", [(2100, 2112), (33001, 33024), (70001, 70016)])
@pytest.mark.parametrize("kind", ["wide", "near", "below", "above", "forced"])
def test_evict_selection_of_unusual_weights(L, cap, kind):
    """Weights of every size and sign, many within 2^-18 of each other, all
    below 2^-24 or above 2^8; and no choice at all."""
    r = Rig("e4m3", "bf16", B=1, H=2, D=64, cap=cap)
    k, v = r.kv(L)
    r.c.append(0, k.cuda(), v.cuda())
    x = torch.rand(2, cap, generator=r.g)
    w = {"wide": torch.randn(2, cap, generator=r.g) * torch.exp2(x * 250 - 140), "near": 1 + x * 2.0 ** -15,
         "below": x * 2.0 ** -30 - 2.0 ** -32, "above": 300 + x * 1e30, "forced": x}[kind]
    r.c.weights.view(2, cap).copy_(w)
    keep, sink, recent = (L // 5, L // 5 - 40, 40) if kind == "forced" else (L // 3, 4, 30)
    pos = r.c.evict(keep, sink, recent).positions.view(2, -1).cpu()
    for h in range(2):
        order = w[h, :L].double()
        order[:sink] = order[L - recent:] = math.inf
        rank = torch.sort(order, stable=True, descending=True)[1][:keep]
        assert torch.equal(pos[h, :keep].long(), torch.sort(rank)[0])


@pytest.mark.parametrize("L,cap", [(139_999, 140_000), (262_145, 262_176), (301_003, 301_024)])
@pytest.mark.parametrize("kind", ["random", "zero", "few", "levels"])
def test_evict_selection_of_many_parts(L, cap, kind):
    """More than sixteen parts, and parts of more than one tile."""
    r = Rig("e4m3", "bf16", B=1, H=2, D=64, cap=cap)
    c = r.c
    c.codes.zero_()
    c.scales.zero_()
    c.tail.zero_()
    c.positions.view(2, cap).copy_(torch.arange(cap, dtype=torch.int32).expand(2, -1))
    c.lengths.fill_(L)
    w = torch.rand(2, cap, generator=r.g)
    w = {"random": w, "zero": w * 0, "few": (w < 0.01).float(), "levels": (w * 40).floor()}[kind]
    c.weights.view(2, cap).copy_(w)
    keep, sink, recent = L // 7, 5, 77
    to = c.evict(keep, sink, recent)
    pos = to.positions.view(2, -1).cpu()
    assert to.lengths.tolist() == [[keep]]
    for h in range(2):
        order = w[h, :L].double()
        order[:sink] = order[L - recent:] = math.inf
        rank = torch.sort(order, stable=True, descending=True)[1][:keep]
        assert torch.equal(pos[h, :keep].long(), torch.sort(rank)[0])
        assert torch.equal(to.weights.view(2, -1)[h, :keep].cpu(), w[h, pos[h, :keep].long()])


def test_evict_parts_of_uneven_sequences():
    """Sequences that end in the first, a later and no part, one that keeps
    everything; more layers than one."""
    r = Rig("e4m3", "bf16", B=4, H=1, D=64, cap=50016, layers=2, layer=1)
    new = [50000, 9000, 0, 300]
    k, v = r.kv(50000)
    r.c.append(1, k.cuda(), v.cuda(), ints(new))
    w = torch.rand(4, 1, 50016, generator=r.g)
    r.c.weights.view(2, 4, 1, -1)[1] = w.cuda()
    to = rq.BlockCache(*r.c.shape, 512, weights=True)
    r.c.evict(500, 3, 20, into=to)
    assert to.lengths.tolist() == [[0] * 4, [500, 500, 0, 300]]
    pos = to.positions.view(2, 4, 512)[1].cpu()
    for b, L in enumerate(new):
        order = w[b, 0, :L].double()
        order[:3] = order[max(0, L - 20):] = 9.0
        want = torch.sort(torch.topk(order, min(L, 500))[1])[0]
        assert torch.equal(pos[b, :min(L, 500)].long(), want)


# ----------------------------------------------------------- used together
@both
def test_serving_run(fmt):
    """Padded prompts, decoded tokens that gather weight, an eviction when the
    cache is full, more tokens over the shrunk cache."""
    r = Rig(fmt, "bf16", B=3, G=2, D=128, cap=160)
    new = [120, 47, 90]
    k, v = r.kv(120, new)
    q = r.randn(3, 4, 120, 128).to(r.dt)
    for b, m in enumerate(new):
        q[b, :, m:] = math.nan
    before = np.zeros_like(r.weights())
    o = r.c.step(0, k.cuda(), v.cuda(), q.cuda(), torch.full(q.shape, 7.5, dtype=r.dt, device="cuda"),
                 ints(new), accumulate=True)
    r.took(k, v, new)
    r.compare(q, o, new, accumulate=True, before=before)
    for turn in range(2):
        for _ in range(30):
            k, v = r.kv(1)
            q = r.randn(3, 4, 1, 128).to(r.dt)
            before = np.nan_to_num(r.weights())
            o = r.c.step(0, k.cuda(), v.cuda(), q.cuda(), accumulate=True)
            r.took(k, v)
            r.compare(q, o, accumulate=True, before=before)
            r.check()
        if turn == 0:
            r = evict(r, 64, 4, 16)
    assert r.lengths() == [94, 94, 94]
    assert [u[0].pos[-1] for u in r.u] == [179, 106, 149]


def test_captured_step_follows_the_lengths():
    """One captured decode step, replayed: lengths, blocks, weights move on."""
    r = Rig("int8", "bf16", B=2, cap=256)
    r.append(60, [60, 13])
    sk, sv = (torch.zeros(2, 2, 1, 128, dtype=r.dt, device="cuda") for _ in range(2))
    sq = torch.zeros(2, 4, 1, 128, dtype=r.dt, device="cuda")
    so = torch.zeros(2, 4, 1, 128, device="cuda")
    ws = torch.empty(rq.rq_block_attention_workspace(r.c.desc, 1, 256, True), dtype=torch.uint8, device="cuda")

    def step():
        past = r.c.lengths[0]
        rq.rq_block_append(r.c.desc, 0, past, sk, sv)
        rq.rq_block_attention(r.c.desc, 0, past, sq, so, ws, accumulate=True)
        r.c.lengths[0] += 1
    lengths = r.c.lengths.clone()
    keep = [t.clone() for t in (r.c.codes, r.c.scales, r.c.tail, r.c.positions, r.c.weights)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    r.c.lengths.copy_(lengths)
    for t, old in zip((r.c.codes, r.c.scales, r.c.tail, r.c.positions, r.c.weights), keep):
        t.copy_(old)
    for turn in range(70):
        k, v = r.kv(1)
        q = r.randn(2, 4, 1, 128).to(r.dt)
        sk.copy_(k)
        sv.copy_(v)
        sq.copy_(q)
        before = np.nan_to_num(r.weights())
        graph.replay()
        torch.cuda.synchronize()
        r.took(k, v)
        r.compare(q, so, accumulate=True, before=before)
    r.check()


def graph_of(call):
    """call(), captured after nothing has run but what it needs."""
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


def test_captured_steps_share_the_cache_with_eager_ones():
    """Two captured steps (one token, three tokens) and eager calls take turns
    on one BlockCache: its workspace grows between the replays, its host bound
    is that of the first captures."""
    r = Rig("e4m3", "bf16", B=2, cap=512)
    r.append(70, [70, 33])
    runs = {}
    for n in (1, 3):
        k, v = (torch.zeros(2, 2, n, 128, dtype=r.dt, device="cuda") for _ in range(2))
        q = torch.zeros(2, 4, n, 128, dtype=r.dt, device="cuda")
        runs[n] = (k, v, q) + graph_of(lambda: r.c.step(0, k, v, q, accumulate=True))
    assert r.c.lengths.tolist() == [[70, 33]]
    held = []                                   # memory that the allocator hands out again
    for turn in range(12):
        for n in (1, 3, 40 if turn % 3 == 2 else 2):
            k, v = r.kv(n)
            q = r.randn(2, 4, n, 128).to(r.dt)
            before = np.nan_to_num(r.weights())
            if n in runs:
                sk, sv, sq, graph, o = runs[n]
                sk.copy_(k)
                sv.copy_(v)
                sq.copy_(q)
                graph.replay()
            else:
                o = r.c.step(0, k.cuda(), v.cuda(), q.cuda(), accumulate=True)
                held.append(torch.full((1 << 20,), math.nan, device="cuda"))
            torch.cuda.synchronize()
            r.took(k, v)
            r.compare(q, o, accumulate=True, before=before)
    assert not any((~h.isnan()).any() for h in held)
    assert r.c.lengths.tolist() == [r.lengths()] and r.c.bound == [512]
    r.check()
    q = r.randn(2, 4, 1, 128).to(r.dt)
    r.compare(q, r.c.attention(0, q.cuda()))
    with pytest.raises(ValueError):
        r.c.append(0, *(x.cuda() for x in r.kv(512 - r.lengths()[0] + 1)))
    r.append(512 - r.lengths()[0])
    r.check()


@pytest.mark.parametrize("n", [1, 3, 20])
@pytest.mark.parametrize("separate", [False, True])
@pytest.mark.parametrize("padded", [False, True])
def test_captured_step_stops_at_the_capacity(n, separate, padded):
    """Replays that reach the capacity: the tokens that fit attend as they would
    in an eager call, the others neither answer nor add weight."""
    r = Rig("e4m3", "bf16", B=4, cap=64)
    r.append(60, [60, 59, 0, 31])
    given = [n, max(n - 1, 0), n, 1] if padded else [n] * 4
    k, v = (torch.zeros(4, 2, n, 128, dtype=r.dt, device="cuda") for _ in range(2))
    q = torch.zeros(4, 4, n, 128, dtype=r.dt, device="cuda")
    new_len = ints(given) if padded else None
    out = torch.zeros(4, 4, n, 128, device="cuda")

    def call():
        if not separate:
            return r.c.step(0, k, v, q, out, new_len, accumulate=True)
        r.c.append(0, k, v, new_len)
        return r.c.attention(0, q, out, new_len, accumulate=True)
    graph, o = graph_of(call)
    for turn in range(7):
        hk, hv = r.kv(n)
        hq = r.randn(4, 4, n, 128).to(r.dt)
        k.copy_(hk)
        v.copy_(hv)
        q.copy_(hq)
        out.fill_(7.5)
        fits = [min(m, 64 - L) for m, L in zip(given, r.lengths())]
        before = np.nan_to_num(r.weights())
        graph.replay()
        torch.cuda.synchronize()
        r.took(hk, hv, fits)
        r.compare(hq, o, fits, accumulate=True, before=before)
        assert r.c.lengths.tolist() == [r.lengths()]
    r.check()
    assert r.lengths()[0] == 64
    # the rows that a call makes for itself hold zeros for such tokens
    graph, o = graph_of(lambda: r.c.step(0, k, v, q, None, new_len))
    for turn in range(2):
        o.fill_(7.5)
        fits = [min(m, 64 - L) for m, L in zip(given, r.lengths())]
        graph.replay()
        torch.cuda.synchronize()
        r.took(hk, hv, fits)
        for b in range(4):
            assert (o[b, :, fits[b]:] == 0).all() and (o[b, :, :fits[b]] != 7.5).all()
    # an eager call afterwards: the tokens handed last, of which these fitted
    o = r.c.attention(0, q, out.fill_(7.5), new_len)
    r.compare(hq, o, fits)
    # lengths taken back by the caller and an eager append: all of it fits again
    for b in range(4):
        for h in range(2):
            u = r.u[b][h]
            u.__init__(u.fmt, u.D, u.narrow)
    r.c.lengths.zero_()
    hk, hv = r.kv(5)
    r.append(5, kv=(hk, hv))
    hq = r.randn(4, 4, 5, 128).to(r.dt)
    r.compare(hq, r.c.attention(0, hq.cuda(), torch.full((4, 4, 5, 128), 7.5, device="cuda")))


def test_advance():
    """Lengths as the append that drops tokens leaves them, out of range and all."""
    c = rq.BlockCache(rq.RQ_INT8, rq.RQ_BF16, 1, 300, 1, 1, 64, 64).desc
    rng = np.random.default_rng(0)
    for n, given in ((1, False), (64, False), (9, True)):
        old, new = rng.integers(-3, 70, 300), rng.integers(-2, 12, 300)
        old[:4] = [-2 ** 31, 2 ** 31 - 1, 64, 0]
        x = [ints(old)] + [torch.full((300,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
        rq.rq_block_advance(c, x[0], n, ints(new) if given else None, *x[1:])
        past = old.clip(0, 64)
        asked = new.clip(0, n) if given else np.full(300, n)
        fit = np.minimum(asked, 64 - past)
        for got, want in zip(x, (past + fit, past, fit, asked - fit)):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
        lengths = ints(old)
        rq.rq_block_advance(c, lengths, n, ints(new) if given else None)
        assert torch.equal(lengths, x[0])
    with pytest.raises(ValueError):
        rq.rq_block_advance(c, None, 1)
    with pytest.raises(ValueError):
        rq.rq_block_advance(c, lengths, 1, past=lengths[:4])


@pytest.mark.parametrize("n", [1, 3])
def test_eviction_after_dropped_tokens(n):
    """The last tokens stay the last: in the smaller cache, too, those that did
    not fit are left out of what follows; the next append has room for all."""
    r = Rig("int8", "bf16", cap=64)
    r.append(63, [63, 20])
    k, v = (torch.zeros(2, 2, n, 128, dtype=r.dt, device="cuda") for _ in range(2))
    graph, _ = graph_of(lambda: r.c.append(0, k, v))
    for turn in range(2):
        hk, hv = r.kv(n)
        k.copy_(hk)
        v.copy_(hv)
        fits = [min(n, 64 - L) for L in r.lengths()]
        graph.replay()
        r.took(hk, hv, fits)
    assert fits == [0, n]
    to = evict(r, 40, 4, 16)
    q = r.randn(2, 4, n, 128).to(r.dt)
    out = torch.full((2, 4, n, 128), 7.5, device="cuda")
    to.compare(q, to.c.attention(0, q.cuda(), out), fits)
    to.append(3)
    to.check()
    q = r.randn(2, 4, 3, 128).to(r.dt)
    to.compare(q, to.c.attention(0, q.cuda()))


def test_captured_attention_and_eviction():
    """A graph that attends, weighs and evicts, replayed over a cache that
    grows by eager calls in between."""
    r = Rig("int8", "fp16", B=2, cap=512)
    to = Rig("int8", "fp16", B=2, cap=96)
    r.append(50)
    q = torch.zeros(2, 4, 1, 128, dtype=r.dt, device="cuda")
    r.c.attention(0, q, accumulate=True)

    def call():
        o = r.c.attention(0, q, accumulate=True)
        r.c.evict(90, into=to.c)
        return o
    graph, o = graph_of(call)
    r.c.weights.view(2, 2, 512)[:, :, :50] = 0.0
    for turn in range(5):
        x = r.randn(2, 4, 1, 128).to(r.dt)
        q.copy_(x)
        before = np.nan_to_num(r.weights())
        graph.replay()
        torch.cuda.synchronize()
        r.compare(x, o, accumulate=True, before=before)
        want = r.c.evict(90)
        kept = min(r.lengths()[0], 90)
        assert to.c.lengths.tolist() == want.lengths.tolist() == [[kept] * 2] and to.c.bound == [96]
        assert torch.equal(to.c.positions.view(4, 96)[:, :kept], want.positions.view(4, 96)[:, :kept])
        assert torch.equal(to.c.codes.view(8, 96, 128)[:, :kept // 32 * 32], want.codes.view(8, 96, 128)[:, :kept // 32 * 32])
        r.append(60)


def test_padding_does_not_use_up_the_capacity():
    r = Rig("int8", "bf16", cap=96)
    for new in ([20, 3], [1, 20], [0, 17], [10, 9], [12, 0]):
        r.append(20, new)
    r.check()
    assert r.c.lengths.tolist() == [[43, 49]]
    with pytest.raises(ValueError):
        r.append(60, [1, 1])          # 49 + 60 rows, whatever they hold


def test_attention_of_more_padded_rows_than_the_cache_holds():
    r = Rig("int8", "bf16", cap=96)
    r.append(5, [5, 3])
    for n in (8, 90):
        q = r.randn(2, 4, n, 128).to(r.dt)
        o = torch.full(q.shape, 7.5, device="cuda")
        r.compare(q, r.c.attention(0, q.cuda(), o, ints([5, 2])), [5, 2])


def test_refused_attention_leaves_the_step_s_tokens():
    r = Rig("int8", "bf16", cap=64, weights=False)
    r.append(40)
    k, v = r.kv(20)
    q = torch.zeros(2, 4, 20, 128, dtype=r.dt, device="cuda")
    with pytest.raises(rq.RQError):
        r.c.step(0, k.cuda(), v.cuda(), q, accumulate=True)       # it keeps no weights
    r.took(k, v)
    assert r.c.lengths.tolist() == [[60, 60]] and r.c.bound == [60]
    q = r.randn(2, 4, 1, 128).to(r.dt)
    r.compare(q, r.c.attention(0, q.cuda()))


def test_another_stream_and_shared_workspace_in_order():
    r = Rig("e4m3", "bf16", cap=256)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        k, v = r.kv(200)
        dk, dv = k.cuda(), v.cuda()
    r.c.append(0, dk, dv, stream=side)
    r.took(k, v)
    q = r.randn(2, 4, 1, 128).to(r.dt)
    with torch.cuda.stream(side):
        dq = q.cuda()
        o = torch.empty(q.shape, device="cuda")
    o = r.c.attention(0, dq, o, stream=side)
    side.synchronize()
    r.compare(q, o)
    to = r.c.evict(50, stream=side)
    side.synchronize()
    assert to.lengths.tolist() == [[50, 50]]


def test_a_new_cache_is_ready_for_any_stream(monkeypatch):
    """The constructor waits for all that it clears: nothing is left on its
    stream, however late, when it returns."""
    held = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (4, 12) for _ in range(64)]
    del held                                    # memory that the allocator hands out again
    make = rq.make_block_cache

    def slow(*a, **kw):
        c = make(*a, **kw)
        if kw:
            torch.cuda._sleep(100_000_000)      # what follows on the stream comes late
        return c
    monkeypatch.setattr(rq, "make_block_cache", slow)
    c = rq.BlockCache(rq.RQ_INT8, rq.RQ_BF16, 2, 2, 1, 1, 64, 64)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        copies = [x.clone() for x in (c.lengths, c._last)]
    side.synchronize()
    late = not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert late and all((x == 0).all() for x in copies)


def test_python_refusals():
    r = Rig("int8", "bf16", cap=64)
    r.append(40)
    k, v = (x.cuda() for x in r.kv(2))
    past = ints([40, 40])
    with pytest.raises(ValueError):
        r.c.append(0, *(x.cuda() for x in r.kv(25)))              # 40 + 25 > 64
    for bad in (k.half(), k[:, :1], k[..., :64], k.cpu(), k.transpose(2, 3), k[0]):
        with pytest.raises(ValueError):
            rq.rq_block_append(r.c.desc, 0, past, bad, v)
    for bad in (None, past.long(), past[:1], past.cpu(), torch.stack([past, past], 1)[:, 0]):
        with pytest.raises(ValueError):
            rq.rq_block_append(r.c.desc, 0, bad, k, v)
    q = torch.zeros(2, 4, 1, 128, dtype=r.dt, device="cuda")
    o = torch.zeros_like(q)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for kw in (dict(q=q.half()), dict(q=q[:, :2]), dict(out=o[:1].expand(2, -1, -1, -1)), dict(out=o.double()), dict(out=o[:1]), dict(ws=ws.cpu()),
               dict(ws=ws[::2]), dict(slopes=torch.zeros(3, device="cuda")), dict(slopes=torch.zeros(4)),
               dict(new_len=past.long())):
        a = dict(q=q, out=o, ws=ws)
        a.update(kw)
        with pytest.raises(ValueError):
            rq.rq_block_attention(r.c.desc, 0, past, **a)
    for kw in (dict(window=-1), dict(cap=-1.0), dict(scale=math.nan), dict(max_tokens=100), dict(ws=ws[:16])):
        with pytest.raises(rq.RQError):
            rq.rq_block_attention(r.c.desc, 0, past, **{**dict(q=q, out=o, ws=ws, accumulate=True), **kw})
    with pytest.raises(ValueError):
        rq.make_block_cache(*r.c.shape, 128, codes=r.c.codes)      # too small
    with pytest.raises(rq.RQError):
        r.c.evict(10, n_sink=8, n_recent=8)
