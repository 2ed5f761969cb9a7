"""The block-scaled cache on the host: sizes, every refusal of its calls (no
kernel is launched: each is validated before), and pins of its oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_06675_amd as rq
from oracle import block

P = 0x10000        # an aligned address that no refused call may touch


def desc(**kw):
    a = dict(format=rq.RQ_INT8, dtype=rq.RQ_BF16, n_layers=2, batch=3,
             n_kv_heads=4, n_q_heads=8, head_dim=128, capacity=96)
    ptrs = {n: P * (i + 1) for i, n in enumerate(
        ("codes", "scales", "tail", "positions", "weights", "counters"))}
    for n in list(kw):
        if n in ptrs:
            ptrs[n] = kw.pop(n)
    a.update(kw)
    c = rq.make_block_cache(**a)
    for n, p in ptrs.items():
        setattr(c, n, p)
    return c


def rows(p=P):
    return rq.RqBlockRows(p, 1, 1, 1)


def query(**kw):
    a = rq.RqBlockQuery(2, 96, P, None, rows(), rows(), rq.RQ_F32, 0.1, 0.0, 0,
                        None, 0)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("D", [64, 128])
def test_sizes(D):
    u = 2 * 3 * 4
    assert rq.rq_block_sizes(desc(head_dim=D)) == (
        u * 2 * 96 * D, u * 2 * 3 * 4, u * 2 * 32 * D * 2, u * 96 * 4, u * 96 * 4, u * 4)


BAD_SHAPES = [
    (dict(format=2), rq.RQ_EINVAL), (dict(dtype=rq.RQ_F32), rq.RQ_EINVAL),
    (dict(head_dim=96), rq.RQ_EUNSUPPORTED), (dict(n_layers=0), rq.RQ_EINVAL),
    (dict(batch=0), rq.RQ_EINVAL), (dict(n_kv_heads=33, n_q_heads=33), rq.RQ_EINVAL),
    (dict(batch=8192), rq.RQ_EUNSUPPORTED), (dict(n_q_heads=6), rq.RQ_EINVAL),
    (dict(n_q_heads=68), rq.RQ_EUNSUPPORTED), (dict(capacity=0), rq.RQ_EINVAL),
    (dict(capacity=100), rq.RQ_EINVAL), (dict(capacity=(1 << 24) + 32), rq.RQ_EINVAL)]


@pytest.mark.parametrize("kw,status", BAD_SHAPES)
def test_shape_refusals(kw, status):
    with pytest.raises(rq.RQError) as e:
        rq.rq_block_sizes(desc(**kw))
    assert e.value.status == status
    L, c = rq.lib(), desc(**kw)
    ok = desc()
    assert L.rq_block_append(C.byref(c), 0, P, 1, None, C.byref(rows()), C.byref(rows()), None) == status
    assert L.rq_block_attention(C.byref(c), 0, C.byref(query()), P, 1 << 40, None) == status
    for pair in ((c, ok), (ok, c)):
        assert L.rq_block_evict(C.byref(pair[0]), C.byref(pair[1]), 0, P, 8, 1, 1, P, P, 1 << 40,
                                None) == status


@pytest.mark.parametrize("kw", [dict(codes=None), dict(scales=None), dict(tail=None),
                                dict(positions=None), dict(codes=P + 8), dict(scales=P + 4),
                                dict(tail=P + 2), dict(positions=P + 4), dict(weights=P + 4),
                                dict(counters=P + 2)])
def test_buffer_refusals(kw):
    c, L = desc(**kw), rq.lib()
    assert L.rq_block_append(C.byref(c), 0, P, 1, None, C.byref(rows()), C.byref(rows()),
                             None) == rq.RQ_EINVAL
    assert L.rq_block_attention(C.byref(c), 0, C.byref(query()), P, 1 << 40, None) == rq.RQ_EINVAL


def test_append_refusals():
    L, c = rq.lib(), desc()

    def call(layer=0, past=P, n=1, k=P, v=P):
        return L.rq_block_append(C.byref(c), layer, past, n, None, C.byref(rows(k)),
                                 C.byref(rows(v)), None)
    for kw in (dict(layer=-1), dict(layer=2), dict(past=None), dict(n=0), dict(n=97),
               dict(k=None), dict(v=None)):
        assert call(**kw) == rq.RQ_EINVAL, kw
        assert rq.rq_last_error()
    assert L.rq_block_append(None, 0, P, 1, None, C.byref(rows()), C.byref(rows()), None) == rq.RQ_EINVAL
    assert L.rq_block_append(C.byref(c), 0, P, 1, None, None, None, None) == rq.RQ_EINVAL


def test_advance_refusals():
    L = rq.lib()
    assert L.rq_block_advance(None, P, 1, None, None, None, None, None) == rq.RQ_EINVAL
    assert L.rq_block_advance(C.byref(desc(capacity=100)), P, 1, None, None, None, None, None) == rq.RQ_EINVAL
    for lengths, n in ((None, 1), (P, 0), (P, 97)):
        assert L.rq_block_advance(C.byref(desc()), lengths, n, None, None, None, None, None) == rq.RQ_EINVAL
        assert rq.rq_last_error()


def test_advance_refuses_overlapping_arrays():
    L, c = rq.lib(), desc()
    for i in range(5):
        for j in range(5):
            if i == j:
                continue
            a = [P * (k + 1) for k in range(5)]
            a[i] = a[j] + (4 if i < j else 8)          # three int32 each
            assert L.rq_block_advance(C.byref(c), a[0], 1, *a[1:], None) == rq.RQ_EINVAL
            assert b"overlap" in L.rq_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n_new=0), -1), (dict(n_new=97, max_tokens=97), -1), (dict(max_tokens=1), -1),
    (dict(max_tokens=97), -1), (dict(past=None), -1), (dict(q=rows(None)), -1),
    (dict(out=rows(None)), -1), (dict(out_dtype=3), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(cap=-1.0), -1), (dict(cap=float("inf")), -1),
    (dict(cap=1e-40), -1), (dict(cap=3e38), -1), (dict(window=-1), -1)])
def test_attention_refusals(kw, status):
    assert rq.lib().rq_block_attention(C.byref(desc()), 0, C.byref(query(**kw)), P, 1 << 40,
                                       None) == status


def test_cap_refusals():
    L, c = rq.lib(), desc()
    for cap in (float("nan"), -1e-30, 2.0 ** 100 * 1.01, 1e38):
        assert L.rq_block_attention(C.byref(c), 0, C.byref(query(cap=cap)), P, 1 << 40, None) == rq.RQ_EINVAL
        assert b"cap" in L.rq_last_error()


def test_attention_workspace_refusals():
    L, c = rq.lib(), desc()
    need = rq.rq_block_attention_workspace(c, 2, 96, True)
    assert need > 0
    q = query(accumulate=1)
    assert L.rq_block_attention(C.byref(c), 0, C.byref(q), P, need - 1, None) == rq.RQ_ESMALLWS
    assert L.rq_block_attention(C.byref(c), 0, C.byref(q), None, need, None) == rq.RQ_EINVAL
    assert L.rq_block_attention(C.byref(c), 0, C.byref(q), P + 8, need, None) == rq.RQ_EINVAL
    assert L.rq_block_attention(C.byref(desc(weights=None)), 0, C.byref(q), P, need, None) == rq.RQ_EINVAL
    assert L.rq_block_attention(C.byref(c), 0, None, P, need, None) == rq.RQ_EINVAL
    assert L.rq_block_attention_workspace(C.byref(c), C.byref(q), None) == rq.RQ_EINVAL


def test_evict_refusals():
    L, src = rq.lib(), desc()
    off = {n: P * (i + 9) for i, n in enumerate(("codes", "scales", "tail", "positions", "weights"))}
    need = rq.rq_block_evict_workspace(src, 40)

    def call(dst=None, s=src, layer=0, lengths=P, keep=40, sink=4, recent=8, out=P, ws=P, size=need):
        d = desc(**{**off, **(dst or {})})
        return L.rq_block_evict(C.byref(s), C.byref(d), layer, lengths, keep, sink, recent, out, ws,
                                size, None)
    for dst in (dict(format=rq.RQ_E4M3), dict(dtype=rq.RQ_F16), dict(n_layers=1), dict(batch=2),
                dict(n_kv_heads=2), dict(n_q_heads=4), dict(head_dim=64), dict(capacity=32),
                dict(codes=src.codes), dict(scales=src.scales), dict(tail=src.tail),
                dict(positions=src.positions), dict(weights=src.weights)):
        assert call(dst) == rq.RQ_EINVAL, dst
    for kw in (dict(layer=2), dict(lengths=None), dict(out=None), dict(keep=0), dict(keep=97),
               dict(sink=-1), dict(recent=0), dict(sink=33), dict(ws=None), dict(ws=P + 4),
               dict(s=desc(weights=None))):
        assert call(**kw) == rq.RQ_EINVAL, kw
    assert call(size=need - 1) == rq.RQ_ESMALLWS


def test_evict_refuses_lengths_that_it_would_overwrite():
    """Every workgroup reads the lengths until the last launch."""
    L, src = rq.lib(), desc()
    dst = desc(**{n: P * (i + 9) for i, n in enumerate(("codes", "scales", "tail", "positions", "weights"))})
    need = rq.rq_block_evict_workspace(src, 40)
    for lengths, new in ((P, P), (P, P + 4), (P + 8, P)):
        assert L.rq_block_evict(C.byref(src), C.byref(dst), 0, lengths, 40, 4, 8, new, P, need,
                                None) == rq.RQ_EINVAL
        assert b"lengths" in L.rq_last_error()


def test_python_refusals_need_no_device():
    with pytest.raises(ValueError):
        rq.make_block_cache(rq.RQ_INT8, rq.RQ_BF16, 1, 1, 1, 1, 64, 32,
                            codes=torch.zeros(1, 1, 1, 2, 32, 64, dtype=torch.int8))


# -------------------------------------------------------------- oracle pins
def test_oracle_e4m3_is_the_published_format():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(block.E4M3_VALUES, want)
    y = np.concatenate([np.random.default_rng(0).normal(size=4000) * 60,
                        block.E4M3_VALUES[:126] + np.diff(block.E4M3_VALUES[:127]) / 2,
                        [0.0, -0.0, 448, -448, 2.0 ** -10, 2.0 ** -11]]).astype(np.float32)
    want = torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(block.e4m3_round(y), want)


@pytest.mark.parametrize("fmt", [block.INT8, block.E4M3])
def test_oracle_quantize(fmt):
    rng = np.random.default_rng(fmt)
    x = rng.normal(size=(32, 64)).astype(np.float32)
    codes, scale = block.quantize(fmt, x)
    back = block.decode(fmt, codes) * scale
    # half a step: of the scale (int8), of the value or of the smallest number (e4m3)
    half = scale / 2 if fmt == block.INT8 else np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -10)
    assert np.all(np.abs(back - x) <= half * (1 + 2.0 ** -20))
    assert np.abs(block.decode(fmt, codes)).max() == (127 if fmt == block.INT8 else 448)
    codes, scale = block.quantize(fmt, np.zeros((32, 64)))
    assert scale == 0 and not codes.any()
    codes, scale = block.quantize(fmt, np.full((32, 64), 1e-38))
    assert scale == 0 and not codes.any()


def test_oracle_unit_attention_and_eviction():
    rng = np.random.default_rng(5)
    u = block.Unit(block.INT8, 64, lambda x: x)
    k, v = rng.normal(size=(2, 70, 64)).astype(np.float32)
    u.append(k, v)
    assert len(u.codes[0]) == 64 and len(u.tail[0]) == 6 and u.length == 70
    q = rng.normal(size=(3, 2, 64)).astype(np.float32)
    out = u.attend(q, 0.125, accumulate=True)
    K, V = (torch.from_numpy(u.values(s)).double() for s in (0, 1))
    for i in range(3):
        n = 68 + i
        want = torch.nn.functional.scaled_dot_product_attention(
            torch.from_numpy(q[i]).double()[:, None], K[None, :n].expand(2, -1, -1),
            V[None, :n].expand(2, -1, -1), scale=0.125)
        np.testing.assert_allclose(out[i], want[:, 0].numpy(), atol=1e-12)
    assert abs(u.weight.sum() - 6) < 1e-12
    w = np.zeros(70)
    w[[9, 20, 30]] = 1.0
    to = u.evict(8, 2, 3, w)
    assert list(to.pos) == [0, 1, 9, 20, 30, 67, 68, 69]
    assert list(u.evict(7, 2, 3, w).pos) == [0, 1, 9, 20, 67, 68, 69]
    np.testing.assert_array_equal(to.tail[0][2], u.values(0)[9])
    assert u.evict(100, 2, 3).length == 70


def test_a_window_needs_no_more_workspace():
    """The size without a window serves every window, whatever the plans."""
    rng = np.random.default_rng(5)
    for _ in range(4000):
        H, G = int(rng.integers(1, 9)), int(rng.integers(1, 17))
        cap = 32 * int(2 ** rng.uniform(0, 12))
        c = desc(batch=int(2 ** rng.uniform(0, 6)), n_kv_heads=H, n_q_heads=H * G, capacity=cap,
                 head_dim=int(rng.choice([64, 128])))
        most = int(rng.integers(1, cap + 1))
        n = int(min(most, 2 ** rng.uniform(0, 13)))
        for acc in (False, True):
            whole = rq.rq_block_attention_workspace(c, n, most, acc)
            for window in (1, int(2 ** rng.uniform(0, 17))):
                assert rq.rq_block_attention_workspace(c, n, most, acc, window) <= whole
