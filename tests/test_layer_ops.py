"""The operators around the cache (include/mikv_layer.h) against plain
implementations in 64 bits (oracle/layer.py)."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import layer as ref
from paper_2402_18096_amd import mikv

D = 128
SCALE = 1 / math.sqrt(128.0)
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
gpu = pytest.mark.gpu


def _np(t):
    return t.detach().double().cpu().numpy()


# -- rotary positions -----------------------------------------------------------------

SCHEMES = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
           dict(scaling="bands", factor=8.0, original_length=8192, low=1.0, high=4.0), dict(scaling="yarn", factor=16.0)]


def _frequencies(rot_dim, **kw):
    """Radians per position from the library's fixed-point fractions of a turn, and the magnitude (host only)."""
    r = mikv.MikvRotary(rot_dim, device="cpu", **kw)
    f = [int(x) % (1 << 64) for x in r.freq.tolist()]
    return np.array(f, dtype=np.float64) * 2.0 ** -64 * 2 * math.pi, r.magnitude


@pytest.mark.parametrize("rot_dim", [2, 20, 64, 128])
@pytest.mark.parametrize("kw", SCHEMES)
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_rotary_frequencies(rot_dim, kw, base):
    if kw.get("scaling") == "ntk" and rot_dim == 2:
        with pytest.raises(mikv.MikvError):
            mikv.MikvRotary(rot_dim, base, device="cpu", **kw)
        return
    got, m = _frequencies(rot_dim, base=base, **kw)
    want, wm = ref.rotary_frequencies(rot_dim, base, **kw)
    # fixed point: half of 2^-62 turns; the oracle's powers: a few ulps
    assert np.all(np.abs(got - want) <= 2 * math.pi * 2.0 ** -62 + 2.0 ** -48 * want)
    assert abs(m - wm) <= 2.0 ** -23


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=130), dict(base=1.0), dict(base=float("nan")),
                                dict(scaling="linear", factor=0.5), dict(scaling="bands", factor=2.0, low=4.0, high=4.0),
                                dict(scaling="yarn", factor=2.0, original_length=0), dict(scaling="other")])
def test_rotary_frequencies_refused(kw):
    with pytest.raises(mikv.MikvError):
        mikv.MikvRotary(device="cpu", **kw)


def _rotary_case(B, T, Hq, Hkv, x, y, packed, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn(B, T, (Hq + 2 * Hkv) * D, device="cuda", generator=g).to(x)
    h = rows.view(B, T, Hq + 2 * Hkv, D).transpose(1, 2)
    xs = [h[:, :Hq], h[:, Hq:Hq + Hkv], h[:, Hq + Hkv:]]
    xs = xs if packed else [t.contiguous() for t in xs]
    return xs, [torch.full(t.shape, float("nan"), dtype=y, device="cuda") for t in xs]


def _check_rotated(x, y, pos, w, m, interleaved, rotate=True):
    """y is x's rotation: two products and a sum in fp32 with sines off by at most
    2^-22 (phase to 2^-25 turns, sine and its product with the magnitude half a step
    each), then one rounding to y's type."""
    want = ref.rotary(_np(x), pos, w, m, interleaved) if rotate else _np(x)
    size = ref.rotary(np.abs(_np(x)), np.zeros_like(pos), w, m, interleaved)
    r = 2 * len(w)
    big = np.abs(size)
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    if rotate:
        both = big[..., ia] + big[..., ib]
        big[..., ia], big[..., ib] = both, both
    tiny = 2.0 ** -25 if y.dtype == torch.float16 else 0.0  # half of the smallest subnormal
    tol = HALF_STEP[y.dtype] * np.abs(want) * (1 + 1e-3) + (2.0 ** -21 * big if rotate else 0.0) + tiny
    err = np.abs(_np(y) - want)
    assert np.all(err <= tol), float((err - tol).max())


@gpu
@pytest.mark.parametrize("x,y", [("float16", "float16"), ("bfloat16", "float16"), ("bfloat16", "bfloat16"),
                                 ("float32", "float16"), ("float32", "float32")])
@pytest.mark.parametrize("rot", [128, 96, 64, 20, 6, 2])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_types_and_parts(x, y, rot, interleaved):
    x, y = getattr(torch, x), getattr(torch, y)
    for B, T, packed in ((2, 1, True), (1, 37, False), (3, 5, True)):
        xs, ys = _rotary_case(B, T, 4, 2, x, y, packed, seed=rot)
        rot_ = mikv.MikvRotary(rot, interleaved=interleaved)
        w, m = _frequencies(rot)
        mikv.mikv_rotary(rot_, xs, ys, pos0=3)
        pos = np.broadcast_to(3 + np.arange(T), (B, T))
        for i in range(3):
            _check_rotated(xs[i], ys[i], pos, w, m, interleaved, rotate=i < 2)


@gpu
@pytest.mark.parametrize("kw", SCHEMES)
def test_rotary_far_and_negative_positions(kw):
    pos = torch.tensor([[0, 1, -1, 4095, 131071, 1048575, -1048575, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    xs, ys = _rotary_case(1, 9, 2, 2, torch.float32, torch.float32, False)
    r = mikv.MikvRotary(128, **kw)
    w, m = _frequencies(128, **kw)
    mikv.mikv_rotary(r, xs, ys, positions=pos)
    # the oracle's angle in 64 bits: 2^31 w is exact to 2^-22 radians only, so the far ends are checked modulo a turn
    phase = np.array([[(int(p) * (int(f) % (1 << 64))) % (1 << 64) for f in r.freq.tolist()] for p in pos[0].tolist()])
    angle = (phase.astype(np.float64) * 2.0 ** -64 * 2 * math.pi)[None, None]
    for t in range(2):
        x = _np(xs[t])
        c, s = np.cos(angle) * m, np.sin(angle) * m
        a, b = x[..., :64], x[..., 64:]
        want = np.concatenate([a * c - b * s, b * c + a * s], axis=-1)
        tol = 2.0 ** -20 * m * np.concatenate([np.abs(a) + np.abs(b)] * 2, axis=-1)
        assert np.all(np.abs(_np(ys[t]) - want) <= tol)
    # turning back by the negative position undoes the turn, and is its transpose
    zs = [torch.empty_like(t) for t in ys]
    mikv.mikv_rotary(r, ys, zs, positions=-pos.clamp(min=-2 ** 31 + 1))
    back = _np(zs[0])[:, :, :8] / (m * m)
    assert np.all(np.abs(back - _np(xs[0])[:, :, :8]) <= 2.0 ** -17 * (1 + np.abs(back).max()))


@gpu
def test_rotary_in_place_strides_and_streams():
    xs, ys = _rotary_case(2, 33, 3, 1, torch.float16, torch.float16, True)
    r = mikv.MikvRotary(64)
    mikv.mikv_rotary(r, xs, ys, pos0=7)
    side = torch.cuda.Stream()
    keep = [t.clone() for t in xs]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mikv.mikv_rotary(r, xs, xs, pos0=7)  # in place, through the projection's strides
    torch.cuda.current_stream().wait_stream(side)
    for a, b, k in zip(xs, ys, keep):
        assert torch.equal(a, b)
    # rows that are not 16-byte aligned, and heads a step apart: the narrow paths, same values
    for shift in (1, 2, 4):
        odd = torch.zeros(2, 33, 5, 200, dtype=torch.float16, device="cuda")[..., shift:shift + D]
        src = odd.transpose(1, 2)[:, ::2]
        src.copy_(keep[0])
        out = torch.empty(2, 3, 33, D, dtype=torch.float16, device="cuda")
        mikv.mikv_rotary(r, [src], [out], pos0=7)
        assert torch.equal(out, ys[0])


@gpu
def test_rotary_captured():
    xs, ys = _rotary_case(2, 9, 4, 4, torch.bfloat16, torch.float16, True)
    r = mikv.MikvRotary(128, interleaved=True)
    pos = torch.arange(18, dtype=torch.int32, device="cuda").view(2, 9).contiguous()
    mikv.mikv_rotary(r, xs, ys, positions=pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mikv.mikv_rotary(r, xs, ys, positions=pos)
    for k in range(3):
        pos.add_(100 * k + 1)
        for x in xs:
            x.copy_(torch.randn_like(x))
        want = [torch.empty_like(y) for y in ys]
        mikv.mikv_rotary(r, xs, want, positions=pos)
        for y in ys:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for y, z in zip(ys, want):
            assert torch.equal(y, z)


# -- spans ------------------------------------------------------------------------------

def _documents(kind, B, T, rng):
    if kind is None:
        return None
    ids = np.zeros((B, T), dtype=np.int32)
    for b in range(B):
        cuts = np.sort(rng.integers(0, T + 1, size=max(1, T // 9 if kind == "many" else 2)))
        ids[b] = np.searchsorted(cuts, np.arange(T), side="right")
        if kind == "padded":
            ids[b, T - int(rng.integers(0, T // 2 + 1)):] = -1
            ids[b, :int(rng.integers(0, T // 4 + 1))] = -5
        if kind == "many" and T > 4:
            ids[b, ::7] = -1
            ids[b, T // 2] = ids[b, 0]
    return ids


def _spans(B, T, documents=None, prefix=None, window=0):
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
    begin = torch.full((B, T), -7, dtype=torch.int32, device="cuda")
    end = torch.full((B, T), -7, dtype=torch.int32, device="cuda")
    mikv.mikv_mask_spans(begin, end, dev(documents), dev(prefix), window)
    return begin, end


def _seen(B, T, documents=None, prefix=None, window=0):
    return np.stack([ref.visible(T, None if documents is None else documents[b], 0 if prefix is None else int(prefix[b]), window)
                     for b in range(B)])


@gpu
@pytest.mark.parametrize("T", [1, 2, 33, 150])
@pytest.mark.parametrize("docs", [None, "few", "many", "padded"])
@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("window", [0, 1, 20, 2 ** 31 - 1])
def test_spans(T, docs, prefix, window):
    rng = np.random.default_rng(T + window % 97)
    B = 3
    ids = _documents(docs, B, T, rng)
    pre = np.array([0, T, T // 3], dtype=np.int32) if prefix else None
    begin, end = _spans(B, T, ids, pre, window)
    j = torch.arange(T, device="cuda")
    got = (j >= begin[..., None]) & (j < end[..., None])
    assert np.array_equal(got.cpu().numpy(), _seen(B, T, ids, pre, window))


@gpu
@pytest.mark.parametrize("T", [1025, 5000, 40001])
def test_spans_long(T):
    """Documents longer and shorter than a thread's stretch, checked against run starts from numpy."""
    rng = np.random.default_rng(T)
    ids = np.repeat(np.arange(T), rng.choice([1, 2, 40, 3000], size=T))[:T].astype(np.int32)[None]
    begin, end = _spans(1, T, ids, np.array([T], dtype=np.int32))
    cut = np.flatnonzero(np.diff(ids[0])) + 1
    starts, ends = np.r_[0, cut], np.r_[cut, T]
    run = np.searchsorted(cut, np.arange(T), side="right")
    assert np.array_equal(begin.cpu().numpy()[0], starts[run])
    assert np.array_equal(end.cpu().numpy()[0], ends[run])


# -- attention of whole prompts -----------------------------------------------------------

def _prompt(B, Hq, Hkv, T, seed=0, packed=False, k_scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if packed:
        rows = torch.randn(B, T, Hq + 2 * Hkv, D, device="cuda", generator=g)
        rows[:, :, Hq:Hq + Hkv] *= k_scale
        rows = rows.half().transpose(1, 2)
        return rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    q = torch.randn(B, Hq, T, D, device="cuda", generator=g).half()
    k = (torch.randn(B, Hkv, T, D, device="cuda", generator=g) * k_scale).half()
    return q, k, torch.randn(B, Hkv, T, D, device="cuda", generator=g).half()


def _slopes(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda")


def _score_error(q, k, cap, slopes, seen):
    """Bound on a score's error [G, T, T]: 128 products summed in fp32 (128 half steps of the sum of their sizes), the
    cap's exponential, reciprocal and products (a few steps of the cap), the bias's and the scaled score's roundings."""
    with np.errstate(invalid="ignore"):
        sizes = np.stack([np.abs(x) @ np.abs(k).T for x in q]) * SCALE
    T = q.shape[1]
    far = np.abs(np.arange(T)[:, None] - np.arange(T)[None, :]) * (0.0 if slopes is None else np.max(slopes))
    e = 2.0 ** -17 * sizes + cap * 2.0 ** -20 + 2.0 ** -22 * (sizes + far)
    return np.where(seen, e, 0.0)


def _check_attention(q, k, v, out, lse, seen, cap=0.0, slopes=None):
    B, Hq, T, _ = q.shape
    G = Hq // k.shape[1]
    Q, K, V, O, L = _np(q), _np(k), _np(v), _np(out), _np(lse)
    for b in range(B):
        for h in range(k.shape[1]):
            sl = None if slopes is None else _np(slopes)[h * G:(h + 1) * G]
            o, z, p = ref.prompt_attention(Q[b, h * G:(h + 1) * G], K[b, h], V[b, h], seen[b], SCALE, cap, sl)
            ds = _score_error(Q[b, h * G:(h + 1) * G], K[b, h], cap, sl, seen[b]).max(axis=-1)  # [G, T]
            # weights: 2^-11 relative each (fp16), 2^-25 absolute below its normal range (a row's largest weight is at least
            # 1 on that scale), and the scores' errors twice (weight and normaliser); output: one rounding
            av = np.abs(np.where(np.isfinite(V[b, h]), V[b, h], 0.0))
            n = seen[b].sum(axis=-1)
            w = (2.0 ** -11 + 2 * ds + n * 2.0 ** -24)[..., None] * (p @ av) + 2.0 ** -25 * (seen[b] @ av)
            tol = 1.05 * (w + 2.0 ** -11 * np.abs(o)) + 2.0 ** -25
            got = O[b, h * G:(h + 1) * G]
            assert np.all(np.abs(got - o) <= tol), (b, h, float(np.abs(got - o).max()))
            gz = L[b, h * G:(h + 1) * G]
            assert np.array_equal(np.isneginf(gz), np.isneginf(z))
            f = np.isfinite(z)
            assert np.all(np.abs(gz[f] - z[f]) <= (ds + 2.0 ** -22 * (1 + np.abs(np.where(f, z, 0))) + n * 2.0 ** -24)[f])


def _run_attention(q, k, v, rules):
    B, Hq, T, _ = q.shape
    out = torch.full((B, T, Hq, D), float("nan"), dtype=torch.float16, device="cuda").transpose(1, 2)
    lse = torch.full((B, Hq, T), float("nan"), dtype=torch.float32, device="cuda")
    mikv.mikv_prompt_attention(q, k, v, out, lse, rules)
    return out, lse


@gpu
@pytest.mark.parametrize("T", [1, 2, 31, 33, 64, 65, 127, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 1)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True), (5.0, True)])
def test_prompt_attention_causal(T, Hq, Hkv, cap, bias):
    q, k, v = _prompt(1, Hq, Hkv, T, seed=T, packed=T % 2 == 1)
    slopes = _slopes(Hq) if bias else None
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(cap, slopes) if cap or bias else None)
    _check_attention(q, k, v, out, lse, _seen(1, T), cap, slopes)


MASKS = [("few", False, 0), ("many", True, 0), ("padded", False, 0), ("padded", True, 40), (None, True, 0), (None, False, 70),
         (None, True, 9), ("few", False, 1)]


@gpu
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 4), (77, 4, 2), (300, 8, 1), (600, 2, 2)])
@pytest.mark.parametrize("docs,prefix,window", MASKS)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, True)])
def test_prompt_attention_masks(T, Hq, Hkv, docs, prefix, window, cap, bias):
    rng = np.random.default_rng(T)
    B = 2
    ids = _documents(docs, B, T, rng)
    pre = np.array([T // 2, T], dtype=np.int32) if prefix else None
    q, k, v = _prompt(B, Hq, Hkv, T, seed=T + 1, k_scale=2.0)
    begin, end = _spans(B, T, ids, pre, window)
    slopes = _slopes(Hq) if bias else None
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(cap, slopes, begin, end))
    _check_attention(q, k, v, out, lse, _seen(B, T, ids, pre, window), cap, slopes)


@gpu
@pytest.mark.parametrize("Hq,Hkv,T", [(64, 8, 65), (32, 8, 385)])
@pytest.mark.parametrize("docs", [None, "few"])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (20.0, True)])
def test_prompts_of_a_full_grid(Hq, Hkv, T, docs, cap, bias):
    """Batches that fill the grid, where a block's eight waves share the rows; a few sequences are checked."""
    B = 16
    ids = _documents(docs, B, T, np.random.default_rng(T))
    q, k, v = _prompt(B, Hq, Hkv, T, seed=T, packed=True)
    begin, end = _spans(B, T, ids, None, 0)
    slopes = _slopes(Hq) if bias else None
    rules = mikv.ScoreRules(cap, slopes, begin, end)
    out, lse = _run_attention(q, k, v, rules)
    scores = torch.full((B, Hkv, T), float("nan"), device="cuda")
    mikv.mikv_prompt_importance(q, k, lse, scores, rules)
    seen = _seen(B, T, ids, None, 0)
    for b in (0, B - 1):
        _check_attention(q[b:b + 1], k[b:b + 1], v[b:b + 1], out[b:b + 1], lse[b:b + 1], seen[b:b + 1], cap, slopes)
        _check_importance(q[b:b + 1], k[b:b + 1], lse[b:b + 1], scores[b:b + 1], seen[b:b + 1], cap, slopes)


@gpu
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 1, 1), (1, 4, 2), (3, 8, 1), (1, 5, 5), (2, 6, 6), (11, 4, 2)])
def test_prompts_of_few_heads(B, Hq, Hkv):
    """Heads that do not fill the eight dies evenly share their blocks out (or not): every row is written once."""
    T = 700
    q, k, v = _prompt(B, Hq, Hkv, T, seed=B)
    out, lse = _run_attention(q, k, v, None)
    scores = torch.full((B, Hkv, T), float("nan"), device="cuda")
    mikv.mikv_prompt_importance(q, k, lse, scores)
    b = B - 1
    _check_attention(q[b:], k[b:], v[b:], out[b:], lse[b:], _seen(1, T))
    _check_importance(q[b:], k[b:], lse[b:], scores[b:], _seen(1, T))
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(scores).all())


@gpu
def test_prompt_attention_any_interval():
    """begin and end of the caller's own, out of range, empty and ahead of the query among them."""
    T, Hq = 333, 4
    rng = np.random.default_rng(5)
    lo = rng.integers(-50, T + 50, size=(2, T)).astype(np.int32)
    hi = (lo + rng.integers(-20, 200, size=(2, T))).astype(np.int32)
    lo[0, :5] = -2 ** 31
    hi[0, :5] = 2 ** 31 - 1
    j = np.arange(T)
    seen = (j >= lo[..., None]) & (j < hi[..., None])
    q, k, v = _prompt(2, Hq, 2, T, seed=9)
    b, e = torch.from_numpy(lo).cuda(), torch.from_numpy(hi).cuda()
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(begin=b, end=e))
    _check_attention(q, k, v, out, lse, seen)
    # one of the two alone
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(begin=b))
    _check_attention(q, k, v, out, lse, (j >= lo[..., None]) & (j <= j[:, None]))
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(end=e))
    _check_attention(q, k, v, out, lse, np.broadcast_to(j < hi[..., None], seen.shape))


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_prompt_attention_masked_rows_hold_anything(bad):
    """NaN and infinities in padding and in another document's keys and values reach no query that does not see them."""
    T = 150
    q, k, v = _prompt(1, 2, 2, T, seed=3)
    ids = np.zeros((1, T), dtype=np.int32)
    ids[0, 40:90], ids[0, 130:] = 1, -1
    k[:, :, 130:], v[:, :, 130:], q[:, :, 130:] = bad, bad, bad
    v[:, :, 20], k[:, 1, 21] = bad, bad  # seen by the first document's later queries
    v[:, :, 60, 5] = bad
    begin, end = _spans(1, T, ids)
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(begin=begin, end=end))
    keep = np.zeros(T, dtype=bool)
    keep[:20], keep[40:60], keep[90:] = True, True, True
    seen = _seen(1, T, ids)
    seen[:, ~keep] = False
    got = out.clone()
    got[:, :, ~torch.from_numpy(keep)] = 0
    z = lse.clone()
    z[:, :, ~torch.from_numpy(keep)] = -float("inf")
    _check_attention(q, k, v, got, z, seen)
    # and a value that is seen is not lost
    o = _np(out)
    assert not np.isfinite(o[0, :, 20:40]).any()
    assert not np.isfinite(o[0, :, 60:90, 5]).any() and np.isfinite(o[0, 0, 60:90, 6]).all()


@gpu
def test_prompt_attention_large_scores():
    """Scores of some hundreds, growing along the sequence, so that the running maximum rises all the way."""
    T = 400
    q, k, v = _prompt(1, 2, 2, T, seed=4)
    k.copy_(q * torch.linspace(0.5, 40, T, device="cuda")[:, None])
    q.copy_(q[:, :, :1].expand_as(q) * 2)
    for rules in (None, mikv.ScoreRules(cap=50.0)):
        out, lse = _run_attention(q, k, v, rules)
        _check_attention(q, k, v, out, lse, _seen(1, T), rules.cap if rules else 0.0)


@gpu
def test_prompt_attention_long_row_sampled():
    """16384 tokens, GQA, window: rows sampled against 64 bits."""
    T, W = 16384, 1500
    q, k, v = _prompt(1, 8, 2, T, seed=6)
    begin, end = _spans(1, T, window=W)
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(cap=30.0, slopes=_slopes(8), begin=begin, end=end))
    for i in (0, 1, 63, 1499, 1500, 8191, 8192, 16383):
        a = max(0, i - W + 1)
        for h in (0, 3, 7):
            s = 30.0 * np.tanh(_np(k)[0, h // 4, a:i + 1] @ _np(q)[0, h, i] * SCALE / 30.0)
            s -= float(_slopes(8)[h]) * (i - np.arange(a, i + 1))
            e = np.exp(s - s.max())
            o = (e / e.sum()) @ _np(v)[0, h // 4, a:i + 1]
            assert np.all(np.abs(_np(out)[0, h, i] - o) <= 2.0 ** -9 * (np.abs(o) + (e / e.sum()) @ np.abs(_np(v)[0, h // 4, a:i + 1])))
            assert abs(float(lse[0, h, i]) - (s.max() + math.log(e.sum()))) <= 1e-4


# -- importance -----------------------------------------------------------------------------

def _check_importance(q, k, lse, scores, seen, cap=0.0, slopes=None):
    B, Hq, T, _ = q.shape
    G = Hq // k.shape[1]
    Q, K, L, S = _np(q), _np(k), _np(lse), _np(scores)
    i, j = np.arange(T)[:, None], np.arange(T)[None, :]
    for b in range(B):
        for h in range(k.shape[1]):
            sl = None if slopes is None else _np(slopes)[h * G:(h + 1) * G]
            ds = _score_error(Q[b, h * G:(h + 1) * G], K[b, h], cap, sl, seen[b])
            want, tol = np.zeros(T), np.zeros(T)
            for g in range(G):
                with np.errstate(invalid="ignore"):
                    s = ref.rule_scores(Q[b, h * G + g] @ K[b, h].T, SCALE, cap, 0.0 if sl is None else float(sl[g]), i - j)
                z = L[b, h * G + g][:, None]
                p = np.where(seen[b], np.exp(np.where(seen[b], s - np.where(np.isfinite(z), z, 0), 0)), 0.0)
                want += p.sum(axis=0)
                # a term: its score's error, and the log-sum-exp's and the difference's roundings in log2 units
                tol += (p * (ds[g] + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(z), z, 0))))).sum(axis=0)
            n = seen[b].sum(axis=0) * G
            tol += n * 2.0 ** -24 * want + 2.0 ** -126 * (1 + n)
            assert np.all(np.abs(S[b, h] - want) <= 1.05 * tol), float(np.abs(S[b, h] - want).max())


def _run_importance(q, k, v, rules):
    _, lse = _run_attention(q, k, v, rules)
    scores = torch.full((q.shape[0], k.shape[1], q.shape[2]), float("nan"), device="cuda")
    mikv.mikv_prompt_importance(q, k, lse, scores, rules)
    return lse, scores


@gpu
@pytest.mark.parametrize("T", [1, 2, 33, 64, 65, 129, 257, 513])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 2, 2), (1, 8, 1), (70, 4, 4)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_prompt_importance_causal(T, B, Hq, Hkv, cap, bias):
    if B > 1 and T > 129:
        B = 2
    q, k, v = _prompt(B, Hq, Hkv, T, seed=T, packed=T % 2 == 1)
    slopes = _slopes(Hq) if bias else None
    lse, scores = _run_importance(q, k, v, mikv.ScoreRules(cap, slopes) if cap or bias else None)
    sub = slice(0, 2)  # the first and last sequence are the ones followed
    pick = lambda t: torch.cat([t[:1], t[-1:]]) if B > 1 else t  # noqa: E731
    _check_importance(pick(q), pick(k), pick(lse), pick(scores), _seen(2, T)[sub][:min(B, 2)], cap, slopes)


@gpu
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 4), (77, 4, 2), (300, 8, 1), (600, 2, 2)])
@pytest.mark.parametrize("docs,prefix,window", MASKS)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, True)])
def test_prompt_importance_masks(T, Hq, Hkv, docs, prefix, window, cap, bias):
    rng = np.random.default_rng(T)
    ids = _documents(docs, 2, T, rng)
    pre = np.array([T // 2, T], dtype=np.int32) if prefix else None
    q, k, v = _prompt(2, Hq, Hkv, T, seed=T + 1, k_scale=2.0)
    begin, end = _spans(2, T, ids, pre, window)
    slopes = _slopes(Hq) if bias else None
    lse, scores = _run_importance(q, k, v, mikv.ScoreRules(cap, slopes, begin, end))
    _check_importance(q, k, lse, scores, _seen(2, T, ids, pre, window), cap, slopes)


@gpu
def test_prompt_importance_any_interval_and_bad_rows():
    T = 333
    rng = np.random.default_rng(5)
    lo = rng.integers(-50, T + 50, size=(2, T)).astype(np.int32)
    hi = (lo + rng.integers(-20, 200, size=(2, T))).astype(np.int32)
    j = np.arange(T)
    q, k, v = _prompt(2, 4, 2, T, seed=9)
    b, e = torch.from_numpy(lo).cuda(), torch.from_numpy(hi).cuda()
    lse, scores = _run_importance(q, k, v, mikv.ScoreRules(begin=b, end=e))
    _check_importance(q, k, lse, scores, (j >= lo[..., None]) & (j < hi[..., None]))
    # padding that holds NaN: its scores are 0, the others' untouched
    ids = np.zeros((2, T), dtype=np.int32)
    ids[:, 200:] = -1
    q[:, :, 200:], k[:, :, 200:], v[:, :, 200:] = float("nan"), float("inf"), float("nan")
    begin, end = _spans(2, T, ids)
    lse, scores = _run_importance(q, k, v, mikv.ScoreRules(begin=begin, end=end))
    _check_importance(q, k, lse, scores, _seen(2, T, ids))
    assert not scores[:, :, 200:].any()


@gpu
def test_prompt_importance_without_rules_is_prefill_importance():
    """The causal case agrees with mikv_prefill_importance (both fp32 sums of the same terms), and its mass is G per query."""
    q, k, v = _prompt(2, 8, 2, 700, seed=1)
    lse, scores = _run_importance(q, k, v, None)
    other = torch.empty_like(scores)
    mikv.mikv_prefill_importance(q, k, other)
    assert torch.allclose(scores, other, rtol=2e-5, atol=1e-6)
    assert torch.allclose(scores.sum(-1), torch.full((2, 2), 700.0 * 4, device="cuda"), rtol=2e-5)


@gpu
def test_prompt_calls_captured_and_on_streams():
    T = 130
    q, k, v = _prompt(2, 4, 2, T, seed=2, packed=True)
    ids = torch.from_numpy(_documents("few", 2, T, np.random.default_rng(0))).cuda()
    begin, end = torch.empty_like(ids), torch.empty_like(ids)
    out, lse = torch.empty(2, 4, T, D, dtype=torch.float16, device="cuda"), torch.empty(2, 4, T, device="cuda")
    scores = torch.empty(2, 2, T, device="cuda")
    ws = torch.empty(mikv.mikv_prompt_importance_workspace_size(2, 4, 2, T), dtype=torch.uint8, device="cuda")
    rules = mikv.ScoreRules(30.0, _slopes(4), begin, end)

    def calls():
        mikv.mikv_mask_spans(begin, end, ids)
        mikv.mikv_prompt_attention(q, k, v, out, lse, rules)
        mikv.mikv_prompt_importance(q, k, lse, scores, rules, workspace=ws)

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for n in range(3):
        q.copy_(torch.randn_like(q))
        ids.copy_(torch.from_numpy(_documents("padded", 2, T, np.random.default_rng(n))).cuda())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls()
            want = [t.clone() for t in (out, lse, scores)]
        torch.cuda.current_stream().wait_stream(side)
        for t in (out, lse, scores):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((out, lse, scores), want):
            assert torch.equal(t, w)


# -- refusals (on the CPU: nothing is launched) ----------------------------------------------------

def _code(fn, *args):
    rc = getattr(mikv.lib(), fn)(*args)
    assert rc == 0 or mikv.lib().mikv_last_error()
    return rc


def _prompt_desc(**kw):
    p = mikv.PromptDesc(1, 4, 2, 64, 128, 0.1, 0x1000, 0x1000, 0x1000)
    for n in ("q", "k", "v"):
        getattr(p, n + "_stride")[:] = [64 * 512, 128, 512]
    for name, value in kw.items():
        if name.endswith("_stride"):
            getattr(p, name)[:] = value
        else:
            setattr(p, name, value)
    return p


BAD_PROMPTS = [(dict(batch=0), 1), (dict(tokens=0), 1), (dict(q_heads=3), 1), (dict(kv_heads=0), 1), (dict(q_heads=12, kv_heads=4), 2),
               (dict(q_heads=32, kv_heads=2), 2), (dict(head_dim=64), 2), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1),
               (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(q=0x1008), 1), (dict(k_stride=[0, 0, 4]), 1),
               (dict(q_stride=[-8, 8, 8]), 1), (dict(q_stride=[8, 8, 1 << 23]), 2), (dict(tokens=2 ** 31 - 1), 2)]


@pytest.mark.parametrize("kw,code", BAD_PROMPTS + [(dict(v=None), 1), (dict(v_stride=[1, 8, 8]), 1)])
def test_prompt_attention_refusals(kw, code):
    s = (ctypes.c_int64 * 3)(64 * 512, 128, 512)
    assert _code("mikv_prompt_attention", ctypes.byref(_prompt_desc(**kw)), None, 0x1000, s, None, None) == code


def test_prompt_attention_refuses_bad_outputs_and_rules():
    p, s = ctypes.byref(_prompt_desc()), (ctypes.c_int64 * 3)(64 * 512, 128, 512)
    assert _code("mikv_prompt_attention", None, None, 0x1000, s, None, None) == 1
    assert _code("mikv_prompt_attention", p, None, None, s, None, None) == 1
    assert _code("mikv_prompt_attention", p, None, 0x1002, s, None, None) == 1
    assert _code("mikv_prompt_attention", p, None, 0x1000, None, None, None) == 1
    assert _code("mikv_prompt_attention", p, None, 0x1000, s, 0x1001, None) == 1
    for rules in (mikv.RulesDesc(-1.0), mikv.RulesDesc(float("nan")), mikv.RulesDesc(float("inf")), mikv.RulesDesc(0.0, 0x1001),
                  mikv.RulesDesc(0.0, None, 0x1002), mikv.RulesDesc(0.0, None, None, 0x1003)):
        assert _code("mikv_prompt_attention", p, ctypes.byref(rules), 0x1000, s, None, None) == 1


@pytest.mark.parametrize("kw,code", BAD_PROMPTS)
def test_prompt_importance_refusals(kw, code):
    assert _code("mikv_prompt_importance", ctypes.byref(_prompt_desc(**kw)), None, 0x1000, 0x1000, 0x1000, 1 << 40, None) == code


def test_prompt_importance_refuses_bad_buffers():
    p = ctypes.byref(_prompt_desc(v=None))
    need = mikv.mikv_prompt_importance_workspace_size(1, 4, 2, 64)
    assert need > 0 and mikv.mikv_prompt_importance_workspace_size(1, 4, 2, 0) == 0
    assert _code("mikv_prompt_importance", p, None, None, 0x1000, 0x1000, need, None) == 1
    assert _code("mikv_prompt_importance", p, None, 0x1000, None, 0x1000, need, None) == 1
    assert _code("mikv_prompt_importance", p, None, 0x1000, 0x1000, None, need, None) == 3
    assert _code("mikv_prompt_importance", p, None, 0x1000, 0x1000, 0x1000, need - 1, None) == 3
    assert _code("mikv_prompt_importance", p, None, 0x1000, 0x1000, 0x1008, need, None) == 1


def test_spans_refusals():
    assert _code("mikv_mask_spans", None, None, 1, 4, 0, None, 0x1000, None) == 1
    assert _code("mikv_mask_spans", None, None, 1, 4, 0, 0x1000, None, None) == 1
    assert _code("mikv_mask_spans", None, None, 0, 4, 0, 0x1000, 0x1000, None) == 1
    assert _code("mikv_mask_spans", None, None, 1, 0, 0, 0x1000, 0x1000, None) == 1
    assert _code("mikv_mask_spans", None, None, 1, 4, -1, 0x1000, 0x1000, None) == 1
    assert _code("mikv_mask_spans", 0x1001, None, 1, 4, 0, 0x1000, 0x1000, None) == 1


def test_rotary_refusals():

    def call(n=1, batch=1, tokens=4, head_dim=128, x_type=0, y_type=0, positions=None, freq=0x1000, rot=128, **kw):
        h = (mikv.Heads * 1)()
        h[0].x, h[0].y, h[0].heads, h[0].rotate = 0x1000, 0x2000, 4, 1
        h[0].x_stride[:] = h[0].y_stride[:] = [2048, 512, 128]
        for name, value in kw.items():
            if name.endswith("stride"):
                getattr(h[0], name)[:] = value
            else:
                setattr(h[0], name, value)
        return _code("mikv_rotary", h, n, batch, tokens, head_dim, x_type, y_type, positions, 0, freq, rot, 0, 1.0, None)

    assert call(n=0) == 1 and call(n=4) == 1 and call(batch=0) == 1 and call(tokens=0) == 1
    assert call(head_dim=64) == 2 and call(rot=3) == 1 and call(rot=0) == 1 and call(rot=130) == 1
    assert call(x_type=3, y_type=3) == 1 and call(x_type=0, y_type=1) == 1 and call(x_type=1, y_type=2) == 1
    assert call(freq=None) == 1 and call(freq=0x1004) == 1 and call(positions=0x1002) == 1
    assert call(x=None) == 1 and call(y=None) == 1 and call(heads=0) == 1 and call(heads=70000) == 2
    assert call(x=0x1001) == 1 and call(y=0x2001) == 1 and call(x_type=2, y_type=2, x=0x1002) == 1
    assert call(batch=1 << 13, tokens=1 << 12) == 2
    assert call(x_type=2, y=0x1000) == 1                      # in place between two types
    assert call(y=0x1000, y_stride=[4096, 512, 256]) == 1     # in place with other strides


def test_binding_refusals():
    x = torch.zeros(1, 2, 3, D, dtype=torch.float16)
    with pytest.raises(mikv.MikvError):
        mikv.mikv_prompt_attention(x, x, x, torch.empty_like(x))  # host tensors
    r = mikv.MikvRotary(device="cpu")
    with pytest.raises(mikv.MikvError):
        mikv.mikv_rotary(r, [x], [x, x])
    with pytest.raises(mikv.MikvError):
        mikv.mikv_rotary(r, [x], [x])
    with pytest.raises(mikv.MikvError):
        mikv.mikv_mask_spans(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32))


def test_outputs_whose_rows_share_memory_are_refused():
    p = ctypes.byref(_prompt_desc())
    for stride in ([8192 * 4, 0, 128], [8192 * 4, 8192, 0]):
        assert _code("mikv_prompt_attention", p, None, 0x1000, (ctypes.c_int64 * 3)(*stride), None, None) == 1
    h = (mikv.Heads * 1)()
    h[0].x, h[0].y, h[0].heads, h[0].rotate = 0x1000, 0x2000, 4, 1
    for stride in ([0, 512, 128], [2048, 0, 128], [2048, 512, 0]):
        h[0].x_stride[:], h[0].y_stride[:] = [2048, 512, 128], stride
        assert _code("mikv_rotary", h, 1, 2, 4, 128, 0, 0, None, 0, 0x1000, 128, 0, 1.0, None) == 1
    assert _code("mikv_mask_spans", None, None, 1, (1 << 30) + 1, 0, 0x1000, 0x1000, None) == 2


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv", [(2, 1), (1, 1)])
def test_prompts_of_more_heads_than_a_grid_dimension(Hq, Hkv):
    # one token: it sees itself alone, so out = v, lse = its score, importance = the heads of its group
    B = 70000
    q, k, v = _prompt(B, Hq, Hkv, 1, seed=1)
    out, lse = _run_attention(q, k, v, mikv.ScoreRules(window=1))
    assert torch.equal(out, v.expand(B, Hkv, 1, D).repeat_interleave(Hq // Hkv, 1))
    scores = torch.full((B + 8, Hkv, 1), -1.0, device="cuda")
    mikv.mikv_prompt_importance(q, k, lse, scores[:B], mikv.ScoreRules(window=1))
    # exp2(s - lse) of the same fp32 score: lse in and out of log2 units and the difference are three roundings of
    # numbers below 16, 2^-21 each, two exponentials half a step or a whole one off: under 4e-6 for two heads
    assert float((scores[:B] - Hq // Hkv).abs().max()) <= 4e-6 and bool((scores[B:] == -1.0).all())


def test_packed_descriptors_have_the_mirrors_layout():
    h = mikv.Heads.from_buffer_copy(mikv._HEADS.pack(16, 32, 1, 2, 3, 4, 5, 6, 7, 1))
    assert (h.x, h.y, list(h.x_stride), list(h.y_stride), h.heads, h.rotate) == (16, 32, [1, 2, 3], [4, 5, 6], 7, 1)
    p = mikv.PromptDesc.from_buffer_copy(mikv._PROMPT.pack(1, 2, 3, 4, 128, 0.5, 16, 32, 0, *range(9)))
    assert (p.batch, p.q_heads, p.kv_heads, p.tokens, p.head_dim, p.scale, p.q, p.k, p.v) == (1, 2, 3, 4, 128, 0.5, 16, 32, None)
    assert [*p.q_stride, *p.k_stride, *p.v_stride] == list(range(9))


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    x = torch.zeros(1, 2, 3, D, dtype=torch.float16, device="cuda")
    spans = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    lse, scores = torch.zeros(1, 2, 3, device="cuda"), torch.zeros(1, 2, 3, device="cuda")
    rotary = mikv.MikvRotary()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 7)
    for call in (lambda: mikv.mikv_rotary(rotary, [x], [x]), lambda: mikv.mikv_mask_spans(spans, spans),
                 lambda: mikv.mikv_prompt_attention(x, x, x, x), lambda: mikv.mikv_prompt_importance(x, x, lse, scores, workspace=spans)):
        with pytest.raises(mikv.MikvError, match="current device"):
            call()


def test_every_declared_layer_symbol_is_bound():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mikv_layer.h")).read()
    names = set(re.findall(r"^(?:int|size_t) (mikv_\w+)\(", text, re.M))
    assert names == set(mikv.LAYER_EXPORTS)
    for n in names:
        assert hasattr(mikv.lib(), n)
