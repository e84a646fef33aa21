"""Decode attention and decode steps under score rules, and a layer's whole
sequence (projection rows -> rotary -> prompt attention -> cache -> steps)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import layer as ref
from paper_2402_18096_amd import mikv, workloads
from tests import parity
from tests.parity import Lockstep, np16

gpu = pytest.mark.gpu

BASE = workloads.WORKLOADS["tiny"].with_(batch=2, q_heads=2, kv_heads=2, context=700, steps=3)
FORMATS = [dict(hi_bits=16, lo_bits=2), dict(hi_bits=8, lo_bits=4, group=64), dict(hi_bits=16, lo_bits=3, group=64),
           dict(hi_bits=4, lo_bits=2), dict(hi_bits=8, lo_bits=2, group=128), dict(hi_bits=16, lo_bits=8),
           dict(hi_bits=16, lo_bits=4), dict(hi_bits=8, lo_bits=8), dict(hi_bits=8, lo_bits=3), dict(hi_bits=16, lo_bits=0),
           dict(hi_bits=16, lo_bits=2, balanced=True, q_outlier_channels=4, q_outlier_scale=10.0),
           dict(hi_bits=8, lo_bits=4, balanced=True)]
RULES = {"cap": dict(cap=20.0), "bias": dict(bias=True), "begin": dict(begin=(130, 640)), "window": dict(window=90),
         "all": dict(cap=20.0, bias=True, begin=(0, 333), window=500), "hidden": dict(begin=(10 ** 6, 5), bias=True)}


class RuledLockstep(Lockstep):
    """Lockstep with the decoder's steps and the oracle's attention under score rules."""

    def __init__(self, wl, steps, cap=0.0, bias=False, begin=None, window=0, fused=False):
        super().__init__(wl, steps, fused)
        slopes = None
        if bias:
            slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / wl.q_heads) for h in range(wl.q_heads)], device="cuda")
        first = None if begin is None else torch.tensor(begin, dtype=torch.int32, device="cuda")
        self.rules = mikv.ScoreRules(cap, slopes, first, None, window)
        H = wl.n_heads
        b = np.zeros(H, int) if begin is None else np.repeat(begin, wl.kv_heads)
        sl = None if slopes is None else np.tile(slopes.cpu().numpy().reshape(wl.kv_heads, wl.group_size), (wl.batch, 1))
        self.orc.attend = lambda q, scale, bal=None: tuple(
            x.astype(np.float32) for x in ref.decode_attention(self.orc, q, scale, b, cap, sl, window, bal))

    def prefill(self):
        super().prefill()
        self.dec.step_rules = self.rules


@gpu
@pytest.mark.parametrize("rules", RULES)
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: "-".join(str(v) for v in f.values()))
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_decode_under_rules(rules, fmt, G):
    run = RuledLockstep(BASE.with_(q_heads=2 * G, seed=BASE.seed + G, **fmt), 2, **RULES[rules])
    run.prefill()
    for t in range(2):
        run.step(t)
    assert int(run.dec.cache.status.item()) == 0


@gpu
@pytest.mark.parametrize("lo", [2, 3, 4])
def test_decode_under_rules_per_channel_keys(lo):
    wl = BASE.with_(lo_bits=lo, key_block=64, window=64, ratio_den=10)
    run = RuledLockstep(wl, 2, **RULES["all"])
    run.prefill()
    for t in range(2):
        run.step(t)


@gpu
@pytest.mark.parametrize("context", [1, 31, 129, 2500])
@pytest.mark.parametrize("G", [1, 4])
def test_decode_under_rules_lengths(context, G):
    wl = BASE.with_(context=context, q_heads=2 * G, ratio_den=2, window=16)
    run = RuledLockstep(wl, 2, cap=10.0, bias=True, begin=(0, context // 3))
    run.prefill()
    for t in range(2):
        run.step(t)


@gpu
@pytest.mark.parametrize("fmt,G", [(FORMATS[0], 1), (FORMATS[0], 4), (FORMATS[1], 2), (FORMATS[9], 1), (FORMATS[10], 8)])
@pytest.mark.parametrize("fused", [False, True])
def test_scored_step_is_the_four_calls(fmt, G, fused):
    wl = BASE.with_(q_heads=2 * G, **fmt)
    kw = dict(RULES["all"], begin=(0, 650))
    a, b = RuledLockstep(wl, 3, fused=fused, **kw), RuledLockstep(wl, 3, fused=fused, **kw)
    a.prefill(), b.prefill()
    for t in range(3):
        x = [y[t].cuda() for y in (a.q, a.kn, a.vn)]
        oa, ob = a.dec.step(*x), b.dec.step_native(*x)
        assert torch.equal(oa, ob)
        for n in ("n_hi", "n_lo", "hi_pos", "map"):
            assert torch.equal(getattr(a.dec.cache, n), getattr(b.dec.cache, n)), n
        n = int(a.dec.cache.n_hi[0])
        assert torch.equal(a.dec.cache.hi_acc[:, :n], b.dec.cache.hi_acc[:, :n])


@gpu
@pytest.mark.parametrize("G", [1, 4])
def test_rules_that_change_nothing(G):
    """A cap far above the scores, slopes of 0 and a window of the whole cache: the unscored results but for tanh's rounding;
    no rules: the same bits."""
    wl = BASE.with_(q_heads=2 * G)
    run = Lockstep(wl, 1)
    run.prefill()
    c, q = run.dec.cache, run.q[0].cuda()
    outs = []
    for rules in (None, mikv.ScoreRules(), mikv.ScoreRules(0.0, torch.zeros(2 * G, device="cuda"), window=10 ** 6),
                  mikv.ScoreRules(1e6)):
        o, ph = torch.empty_like(run.dec.out), torch.empty_like(run.dec.probs_hi)
        mikv.mikv_decode_attention_scored(c, 700, q, o, ph, run.dec.probs_lo, rules)
        outs.append((o, ph[:, :, :int(c.n_hi[0])].clone()))
    plain = torch.empty_like(run.dec.out)
    mikv.mikv_decode_attention(c, 700, q, plain, run.dec.probs_hi, run.dec.probs_lo)
    assert torch.equal(outs[0][0], plain) and torch.equal(outs[1][0], plain)
    # The unscored dot products take 2-bit codes as the deepest fp16 subnormals, with products off by 5e-6: a score
    # is off by e = 5e-6 scale sum |q k|, a probability by a factor of 1 + 2 e (its weight's and the sum's errors), an
    # output by 2 e sum p |v|; the scored ones and the sums' roundings stay within another e.
    tol_o = np.zeros((4, G, 128))
    q_abs = np.abs(np16(run.q[0]).astype(np.float64).reshape(4, G, 128))
    _, p = ref.decode_attention(run.orc, np16(run.q[0]).reshape(4, G, 128), parity.SCALE, np.zeros(4, int))
    worst = 0.0
    for h in range(4):
        kk, vv = (np.abs(x.astype(np.float64)) for x in run.orc.values(h))
        e = 5e-6 * parity.SCALE * (q_abs[h] @ kk.T).max(axis=1)
        tol_o[h] = 3 * e[:, None] * (p[h] @ vv)
        worst = max(worst, 3 * e.max())
    for o, ph in outs[2:]:
        assert np.all(np.abs((o - plain).cpu().numpy().reshape(4, G, 128)) <= tol_o)
        assert torch.allclose(ph, outs[0][1], rtol=worst, atol=1e-12)


@gpu
@pytest.mark.parametrize("hi,lo", [(16, 2), (8, 4), (16, 0)])
@pytest.mark.parametrize("G", [1, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_hidden_tokens_hold_anything(hi, lo, G, bad):
    """Rows placed from NaN or infinities before the first visible position change no bit of the result."""
    T, first = 300, 120
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn(1, 2, T, 128, device="cuda", generator=g).half() for _ in range(2))
    q = torch.randn(1, 2 * G, 128, device="cuda", generator=g).half()
    mask = (torch.rand(1, 2, T, device="cuda", generator=g) < 0.5).to(torch.uint8)
    begin = torch.tensor([first], dtype=torch.int32, device="cuda")
    got = []
    for spoil in (False, True):
        c = mikv.MikvCache(1, 2 * G, 2, 32, hi, lo, T, T, T)
        if spoil:
            k[:, :, 5:first], v[:, :, 5:first] = bad, bad
        mikv.mikv_quantize_kv(c, k, v, 0, None, mask)
        out = torch.empty(1, 2 * G, 128, device="cuda")
        ph, pl = torch.zeros(1, 2 * G, c.cap_hi, device="cuda"), torch.zeros(1, 2 * G, max(1, c.cap_lo), device="cuda")
        mikv.mikv_decode_attention_scored(c, T, q, out, ph, pl if lo else None, mikv.ScoreRules(begin=begin))
        got.append((out, ph, pl))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@gpu
@pytest.mark.parametrize("hi,lo,G", [(16, 2, 1), (16, 2, 2), (16, 2, 8), (16, 3, 1), (8, 4, 4), (4, 2, 2), (16, 8, 8), (16, 0, 4)])
def test_window_over_chunks(hi, lo, G):
    """A window that hides whole chunks of both pools, in a cache of far more capacity than tokens (empty chunks): the cache
    of the window's tokens alone, but for the order of the sums."""
    T, W, cap = 3001, 403, 9000
    g = torch.Generator(device="cuda").manual_seed(hi + lo)
    k, v = (torch.randn(2, 2, T, 128, device="cuda", generator=g).half() for _ in range(2))
    q = torch.randn(2, 2 * G, 128, device="cuda", generator=g).half()
    mask = (torch.rand(2, 2, T, device="cuda", generator=g) < 0.3).to(torch.uint8)
    got = []
    for first, rules in ((0, mikv.ScoreRules(window=W)), (T - W, mikv.ScoreRules(window=cap))):
        n = T - first
        c = mikv.MikvCache(2, 2 * G, 2, 32, hi, lo, cap, cap, cap)
        mikv.mikv_quantize_kv(c, k[:, :, first:].contiguous(), v[:, :, first:].contiguous(), 0, None, mask[:, :, first:].contiguous())
        out = torch.empty(2, 2 * G, 128, device="cuda")
        ph = torch.zeros(2, 2 * G, c.cap_hi, device="cuda")
        pl = torch.zeros(2, 2 * G, c.cap_lo, device="cuda") if lo else None
        mikv.mikv_decode_attention_scored(c, n, q, out, ph, pl, rules)
        probs = torch.empty(2, 2 * G, n, device="cuda")
        mikv.mikv_probs_by_position(c, n, ph, pl, probs)
        got.append((out, probs))
    (out, probs), (want, p) = got
    assert bool((probs[..., :T - W] == 0).all())
    # sums of at most W terms in another order, exponentials and split weights against another maximum: 2^-23 each
    tol = (W + 16) * 2.0 ** -23
    assert bool(((probs[..., T - W:] - p).abs() <= tol * p).all())
    assert float((out - want).abs().max()) <= tol * float(v.abs().max())


@gpu
def test_decode_precision_is_fp32():
    """Probabilities and outputs of an fp16 + 2-bit cache to a few fp32 steps of the scores: capped scores keep the digits of
    scores far below their cap."""
    wl = BASE.with_(q_heads=8, context=900, kv_outlier_scale=2.0)
    run = RuledLockstep(wl, 1, cap=50.0, bias=True)
    run.prefill()
    c = run.dec.cache
    ph, pl, out = run.dec.probs_hi, run.dec.probs_lo, run.dec.out
    mikv.mikv_decode_attention_scored(c, 900, run.q[0].cuda(), out, ph, pl, run.rules)
    sl = np.tile(run.rules.slopes.cpu().numpy().reshape(2, 4), (2, 1))
    o, p = ref.decode_attention(run.orc, np16(run.q[0]).reshape(4, 4, 128), parity.SCALE, np.zeros(4, int), 50.0, sl)
    n_hi, n_lo = c.n_hi.cpu().numpy(), c.n_lo.cpu().numpy()
    got = parity.probs_by_position(c, ph, pl, n_hi, n_lo, c.hi_pos.cpu().numpy(), c.lo_pos.cpu().numpy(), 900)
    assert np.all(np.abs(got - p) <= 2e-5 * p + 1e-12)
    assert np.linalg.norm(out.cpu().numpy().reshape(4, 4, 128) - o) <= 5e-6 * np.linalg.norm(o)


def test_scored_decode_refusals():
    L = mikv.lib()
    c = mikv.CacheDesc()
    for k, v in dict(batch=1, q_heads=4, kv_heads=4, head_dim=128, group=32, hi_bits=16, lo_bits=2, cap_hi=8, cap_lo=32,
                     max_len=16).items():
        setattr(c, k, v)
    for f in ("hi_k", "hi_v", "hi_pos", "hi_acc", "n_hi", "n_lo", "status", "lo_k", "lo_v", "lo_kp", "lo_vp", "lo_pos"):
        setattr(c, f, 0x1000)
    p = ctypes.c_void_p(0x1000)

    def attend(rules, length=4, ws=1 << 30):
        return L.mikv_decode_attention_scored(ctypes.byref(c), length, p, None, 0.1, rules and ctypes.byref(rules), p, p, p, 0, p,
                                              ws, None)

    def step(rules, ws=1 << 30):
        return L.mikv_decode_step_scored(ctypes.byref(c), 4, p, p, p, None, 0.1, rules and ctypes.byref(rules), p, p, p, 1, 1, 0, p,
                                         ws, None, None)

    bad = [mikv.RulesDesc(-1.0), mikv.RulesDesc(float("nan")), mikv.RulesDesc(float("inf")), mikv.RulesDesc(0.0, 0x1002),
           mikv.RulesDesc(0.0, None, 0x1001), mikv.RulesDesc(0.0, None, None, 0x1000), mikv.RulesDesc(0.0, None, None, None, -1)]
    for r in bad:
        assert attend(r) == 1 and step(r) == 1
    good = mikv.RulesDesc(30.0, 0x1000, 0x1000)
    assert attend(good, length=17) == 3 and attend(good, ws=16) == 3 and step(good, ws=16) == 3
    assert attend(None, length=0) == 1


def test_decoder_refuses_masks_of_its_own():
    with pytest.raises(mikv.MikvError):
        mikv.MikvDecoder(BASE, device="cpu", rules=mikv.ScoreRules(begin=torch.zeros(2, dtype=torch.int32)))


# -- a layer's whole sequence ---------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("G,dtype", [(1, torch.float16), (4, torch.bfloat16)])
@pytest.mark.parametrize("masked", [False, True])
def test_layer_sequence(G, dtype, masked):
    """A fused projection's rows through rotary, prompt attention, importance, cache and three steps, against the same in 64
    bits: every token kept in fp16 (ratio 1), so that nothing but roundings lies between them."""
    B, Hkv, T, steps = 2, 2, 200, 3
    Hq = Hkv * G
    wl = BASE.with_(batch=B, q_heads=Hq, kv_heads=Hkv, context=T, steps=steps, ratio_num=1, ratio_den=1, window=16, hi_bits=16,
                    lo_bits=2)
    slopes = torch.tensor([2.0 ** (-h - 1) for h in range(Hq)], device="cuda")
    rotary = mikv.MikvRotary(96, scaling="yarn", factor=4.0)
    dec = mikv.MikvDecoder(wl, fused=True, rotary=rotary, rules=mikv.ScoreRules(25.0, slopes, window=150))
    g = torch.Generator(device="cuda").manual_seed(G)
    rows = torch.randn(B, T + steps, Hq + 2 * Hkv, 128, device="cuda", generator=g).to(dtype)
    heads = rows.transpose(1, 2)
    split = lambda a, z: (heads[:, :Hq, a:z], heads[:, Hq:Hq + Hkv, a:z], heads[:, Hq + Hkv:, a:z])  # noqa: E731
    ids = None
    if masked:
        ids = torch.zeros(B, T, dtype=torch.int32, device="cuda")
        ids[0, :60], ids[1, :70], ids[1, 70:90] = -1, 3, 1
    out = dec.attend_prompt(*split(0, T), documents=ids)
    w, m = ref.rotary_frequencies(96, scaling="yarn", factor=4.0)
    pos = np.broadcast_to(np.arange(T + steps), (B, T + steps))
    x = heads.double().cpu().numpy()
    half = lambda a: a.astype(np.float16).astype(np.float64)  # noqa: E731
    q, k, v = half(ref.rotary(x[:, :Hq], pos, w, m)), half(ref.rotary(x[:, Hq:Hq + Hkv], pos, w, m)), half(x[:, Hq + Hkv:])
    first = [0, 0] if ids is None else [60, 90]
    sl = slopes.cpu().numpy()
    scores = np.zeros((B, Hkv, T))
    for b in range(B):
        seen = ref.visible(T, None if ids is None else ids[b].cpu().numpy(), 0, 150)
        for h in range(Hkv):
            o, _, p = ref.prompt_attention(q[b, h * G:(h + 1) * G, :T], k[b, h, :T], v[b, h, :T], seen, parity.SCALE, 25.0,
                                           sl[h * G:(h + 1) * G])
            scores[b, h] = p.sum(axis=(0, 1))
            got = out[b, :, h * G:(h + 1) * G].double().cpu().numpy().transpose(1, 0, 2)
            # the rotated rows are the same fp16 numbers but for rare ties; weights and output round to fp16
            assert np.linalg.norm(got - o) <= 2e-3 * np.linalg.norm(o)
    c = dec.cache
    n = int(c.n_hi[0])
    assert n == T and np.array_equal(c.hi_pos[0, :n].cpu().numpy(), np.arange(T))
    acc = c.hi_acc[:, :n].cpu().numpy().reshape(B, Hkv, T)
    assert np.allclose(acc, scores, rtol=5e-3, atol=5e-3)
    for t in range(steps):
        args = [y.squeeze(2) for y in split(T + t, T + t + 1)]
        o = dec.step_native(*args).double().cpu().numpy()
        L = T + t + 1
        at = np.arange(L)
        for b in range(B):
            ok = (at >= first[b]) & (at > L - 1 - 150)
            for h in range(Hq):
                s = ref.rule_scores(k[b, h // G, :L] @ q[b, h, L - 1], parity.SCALE, 25.0, sl[h], L - 1 - at)
                p, _ = ref.masked_softmax(s, ok)
                want = p @ v[b, h // G, :L]
                assert np.linalg.norm(o[b, h] - want) <= 2e-3 * np.linalg.norm(want)
    assert int(c.status.item()) == 0
