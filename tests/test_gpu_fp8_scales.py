"""Scales of the 8-bit results where they hang by a thread: sums that cancel, gates far below zero, slopes next to their zero."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc
from paper_2312_17482_amd import binding as mb
from tests.test_gpu_fp8 import BF16, bf16, check_eight, dev, exps, stored, val

pytestmark = pytest.mark.gpu


def act(x, w):
    """(what the operands stand for, the activation's codes and scales)"""
    (xv, xq, xs), (wv, wq, ws) = stored(x), stored(w, 128)
    assert np.array_equal(xv, x) and np.array_equal(wv, w)        # (the operands are exact in 8 bits)
    q, s = mb.mb_geglu_fp8_act(xq, xs, wq, ws)
    hg, inter = x @ w.T, len(w) // 2
    return orc.gelu(hg[:, :inter])[0] * hg[:, inter:], val(q), exps(s), q, s


def octave():
    """Rows whose columns 64, 72, 80 add up to 224 .. 448 in steps of 1/8, less than a window of 2.8e-4 to either side of a
    border: whatever a gate is computed as, some row's value comes to lie beside 448 * 2^e."""
    total = np.arange(224, 448, 0.125)
    first = np.floor(total / 32) * 32
    second = np.floor((total - first) / 2) * 2
    x = np.zeros((len(total), 128))
    x[:, 64], x[:, 72], x[:, 80] = first, second, total - first - second
    return x


def cancelling():
    """h = -2^-8 out of 448 - 448 + 0.0390625 in one group of 8 products and -0.04296875 in another.  The first group keeps 2^-5 at
    the finest, so that h is computed as some -3 * 2^-8."""
    x, w = octave(), np.zeros((256, 128))
    x[:, 0], x[:, 1], x[:, 2], x[:, 8] = 448.0, 448.0, 1.0, 1.0
    w[:128, 0], w[:128, 1], w[:128, 2], w[:128, 8] = 1.0, -1.0, 0.0390625, -0.04296875
    w[128:, [64, 72, 80]] = 1.0
    return x, w


def test_act_of_cancelling_sums_is_the_same_each_time():
    """Which values are looked at again in 64 bits must not hang on which wave comes first."""
    x, w = cancelling()
    _, _, _, q, s = act(x, w)
    for _ in range(20):
        _, _, _, q2, s2 = act(x, w)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s.view(torch.uint8), s2.view(torch.uint8))


def test_act_of_cancelling_sums_stays_finite():
    """Where 64 bits move a value far from what the matrix cores made of it, and the scale with it, what is stored fits that scale:
    the value lies between the exact one and three times it, never beyond e4m3."""
    x, w = cancelling()
    v, q, e, _, _ = act(x, w)
    got = q * np.repeat(np.ldexp(1.0, e), 128, 1)
    assert np.isfinite(q).all()
    ratio = got / v                                               # (GeLU(-3 a) / GeLU(-a) < 3; a rounding is 2^-4)
    assert np.all((ratio >= 1 - 2.0 ** -4) & (ratio <= 3 * (1 + 2.0 ** -4)))
    # a block that was looked at again holds the exact values
    again = np.all(np.abs(ratio - 1) <= 2.0 ** -4, 1)
    print(again.sum(), "tokens looked at again")
    assert again.any() and np.array_equal(e[again], orc.scale_exponents(v)[again])


def test_act_value_beside_a_cancelling_one():
    """One column is computed at the border and is a third of it; the others, just under what is looked at again, need the scale."""
    x, w = cancelling()
    w[1:128], w[129:] = 0.0, 0.0
    w[128] *= -256.0                                              # computed as 333 .. 666
    x[:, 16], x[:, 24] = 16.0, 1.0
    w[1:32, 16], w[129:160, 24] = 1.0, 26.0                       # 416, whose scale is 448's
    v, q, e, _, _ = act(x, w)
    got = q * np.repeat(np.ldexp(1.0, e), 128, 1)
    assert np.all(np.abs(got[:, 1:32] / 416 - 1) <= 2.0 ** -4)


def test_act_a_value_far_below_the_border_does_not_end_the_search():
    """Column 0 of a token is computed beside 448 and is 0.503 of it, a mantissa over 1.75; column 5 is 448 (1 + 2^-17) and computed as
    448: it decides, however early the other one is looked at."""
    x, w = octave(), np.zeros((256, 128))
    x[:, 0], x[:, 1], x[:, 2], x[:, 8] = 448.0, 448.0, 1.0, 1.0
    w[0, 0], w[0, 1], w[0, 2], w[0, 8] = 1.0, -1.0, 0.0390625, -0.046875
    w[128, [64, 72, 80]] = -192.0
    x[:, 16], x[:, 17], x[:, 24] = 16.0, 1.0, 16.0
    w[5, 16], w[5, 17] = 1.0, 2.0 ** -13
    w[128 + 5, 24] = 1.75
    v, q, e, _, _ = act(x, w)
    assert np.array_equal(orc.scale_exponents(v), np.ones((len(x), 1))) and np.all(e == 1)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("h", [-0.75, -0.75390625, -0.7421875, -0.6875, -0.8125, -0.65625, -0.875, 0.5])
def test_gate_backward_scales_beside_the_slopes_zero(h, eight):
    """GeLU' is 0 at -0.7518: blocks whose one gradient meets a gate beside it, da g over all mantissas of bf16."""
    if eight and np.ldexp(np.rint(np.ldexp(abs(h), 4)), -4) != abs(h):
        h = -0.75
    m = 1.0 + np.arange(128) / 128.0
    da, hg = np.zeros((128 * 128, 128)), np.full((128 * 128, 256), h)
    da[:, 5], hg[:, 128:] = np.repeat(m, 128), 0.0
    hg[:, 128 + 5] = np.tile(m, 128)
    if eight:
        hg, hgq, hgs = stored(hg)
    else:
        hgq, hgs = dev(hg, BF16), None
    q, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), hgq, hgs)
    value, slope = orc.gelu(hg[:, :128])
    v = np.concatenate([da * hg[:, 128:] * slope, da * value], 1)
    want, got = orc.scale_exponents(v), exps(s)
    top = np.abs(v).reshape(-1, 2, 128).max(2)
    beside = np.ldexp(448.0, np.floor(np.log2(top / 448.0) + 0.5).astype(int))
    # what 64 bits leave: 4e-10 of the distribution function, of which the slope is a small difference
    clear = np.abs(top / beside - 1) > 1e-8 + 4e-10 * 0.5 / np.abs(slope[0, 0])
    print(h, (got != want).sum(0), "scales of", len(want), "that are not the definition's;", (~clear).sum(), "too near")
    assert (~clear).sum() < 8 and np.array_equal(got[clear], want[clear])
    sc = np.repeat(np.ldexp(1.0, got), 128, 1)
    assert np.all(np.abs(val(q) * sc - v) <= 2.0 ** -4 * (1 + 1e-3) * np.abs(v) + 2.0 ** -10 * sc)


@pytest.mark.parametrize("eight", [False, True])
def test_gate_backward_scales_are_the_definitions(eight):
    """192,000 blocks of ordinary gates, some of them within 7e-5 of a border."""
    T, inter = 12000, 1024
    rng = np.random.default_rng(78)
    da, hg = bf16(rng.standard_normal((T, inter))), rng.standard_normal((T, 2 * inter))
    if eight:
        hg, hgq, hgs = stored(hg)
    else:
        hg = bf16(hg)
        hgq, hgs = dev(hg, BF16), None
    _, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), hgq, hgs)
    value, slope = orc.gelu(hg[:, :inter])
    v = np.concatenate([da * hg[:, inter:] * slope, da * value], 1)
    top = np.abs(v).reshape(T, 16, 128).max(2)
    beside = np.ldexp(448.0, np.floor(np.log2(top / 448.0) + 0.5).astype(int))
    clear = np.abs(top / beside - 1) > 1e-8
    assert clear.sum() > 191980 and (np.abs(top / beside - 1) < 7e-5).sum() >= (1 if eight else 4)   # (values of few bits)
    assert np.array_equal(exps(s)[clear], orc.scale_exponents(v)[clear])


def test_gate_backward_of_large_factors_with_a_small_slope():
    """da g beyond the largest float times a slope that is next to nothing is a finite value, or zero."""
    da, hg = np.zeros((3, 128)), np.zeros((3, 256))
    da[:, 0], hg[:, 128] = 2.0 ** 70, 2.0 ** 70
    hg[:, 0] = [-30.0, -9.0, -12.0]
    q, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), dev(hg, BF16))
    value, slope = orc.gelu(hg[:, :1])
    want = (da[:, :1] * hg[:, 128:129] * slope)[:, 0]
    got = val(q)[:, 0] * np.ldexp(1.0, exps(s)[:, 0])
    assert np.isfinite(val(q)[:, :128]).all() and got[0] == 0.0
    assert np.all(np.abs(got - want)[1:] <= 2.0 ** -4 * (1 + 1e-3) * np.abs(want)[1:])


@pytest.mark.parametrize("mean,xs,ws,low,high", [(5.8, 0.1, 0.3, -6.5, -5.0), (8.5, 0.5, 2.0, -13.0, -5.0)])
def test_act_scales_of_far_negative_gates(mean, xs, ws, low, high):
    """Every gate of 24,000 blocks far below zero, sums of 768 products: an error of h is h^2 times as much of GeLU(h)."""
    T, hidden, inter = 12000, 768, 256
    rng = np.random.default_rng(77)
    x, xq, xsc = stored(1.0 + xs * rng.standard_normal((T, hidden)))
    w = np.concatenate([-(mean / hidden) * (1.0 + ws * rng.standard_normal((inter, hidden))), 0.03 * rng.standard_normal((inter, hidden))])
    w, wq, wsc = stored(w, 128)
    hg = x @ w.T
    h = hg[:, :inter]
    assert h.max() < high and h.min() > low
    v = orc.gelu(h)[0] * hg[:, inter:]
    top = np.abs(v).reshape(T, 2, 128).max(2)
    beside = np.ldexp(448.0, np.floor(np.log2(top / 448.0) + 0.5).astype(int))
    clear = np.abs(top / beside - 1) > 1e-8                       # (GeLU in 64 bits is good to 4e-10)
    _, s = mb.mb_geglu_fp8_act(xq, xsc, wq, wsc)
    wrong = exps(s) != orc.scale_exponents(v)
    print(wrong.sum(), "of", wrong.size, "scales;", (np.abs(top / beside - 1) < 1e-3).sum(), "blocks within 1e-3 of a border")
    assert not wrong[clear].any()


def test_act_beside_one_large_channel():
    """One channel moves every gate to -9: its product outweighs those it is added with, of which it keeps 2^-10.  Values and scales
    are within what that leaves, 7 * 2^-13 of the sums of magnitudes."""
    T, hidden, inter = 3000, 768, 256
    rng = np.random.default_rng(79)
    x, w = rng.standard_normal((T, hidden)), 0.03 * rng.standard_normal((2 * inter, hidden))
    x[:, 5], w[:inter, 5], w[inter:, 5] = 12.0, -0.75, 0.0
    (x, xq, xs), (w, wq, ws) = stored(x), stored(w, 128)
    q, s = mb.mb_geglu_fp8_act(xq, xs, wq, ws)
    hg, eps = x @ w.T, (7 * 2.0 ** -13 + (hidden + 8) * 2.0 ** -24) * (np.abs(x) @ np.abs(w).T)
    h, g = hg[:, :inter], hg[:, inter:]
    value, off = orc.gelu(h)[0], np.abs(orc.gelu(h + eps[:, :inter])[0] - orc.gelu(h)[0])
    assert h.max() < -4 and np.isfinite(val(q)).all()
    check_eight(q, s, value * g, off * (np.abs(g) + eps[:, inter:]) + np.abs(value) * eps[:, inter:] + 5e-5 * np.abs(value * g))


def test_linear_of_cancelling_sums():
    """What a caller gets by asking for fp32 results: sums of fp32, where the others are off by what their groups drop."""
    x, w = cancelling()
    (_, xq, xs), (_, wq, ws) = stored(x), stored(w, 128)
    y, A = x @ w.T, np.abs(x) @ np.abs(w).T
    fine = mb.mb_linear_fp8_fwd(xq, xs, wq, ws, dtype=torch.float32).double().cpu().numpy()
    rough = mb.mb_linear_fp8_fwd(xq, xs, wq, ws).double().cpu().numpy()
    assert np.all(np.abs(fine - y) <= 136 * 2.0 ** -24 * A)
    assert np.all(np.abs(rough - y) <= 136 * 2.0 ** -24 * A + 7 * 2.0 ** -13 * A + 2.0 ** -8 * np.abs(y))
