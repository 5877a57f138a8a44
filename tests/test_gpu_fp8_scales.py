"""Scales of the 8-bit results where they hang by a thread: sums that cancel, gates far below zero, slopes next to their zero; values that
are not finite, and the first and the last scale byte, through the operators."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc
from paper_2312_17482_amd import binding as mb
from tests.test_gpu_fp8 import BF16, E4M3, E8M0, bf16, check_eight, dev, exps, stored, val

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


def test_act_of_what_is_not_finite():
    """NaN in a token, in a weight's row, and sums beyond the largest float: stored as NaN, without a part in the scale."""
    T, hidden, inter = 70, 256, 256
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((T, hidden)), rng.standard_normal((2 * inter, hidden)) * 0.1
    x[4, 130] = np.nan                                            # the token
    w[7, 3], w[inter + 200, 250] = np.nan, np.inf                 # columns 7 and 200
    x[9] *= 2.0 ** 100                                            # h g some 2^200: every column of the token
    x[10, :], x[10, 0] = 0.0, 1e-30
    (xv, xq, xs), (wv, wq, ws) = stored(x), stored(w, 128)
    q, s = mb.mb_geglu_fp8_act(xq, xs, wq, ws)
    hg = xv @ wv.T
    v = orc.gelu(hg[:, :inter])[0] * hg[:, inter:]
    v[9] = np.where(np.abs(v[9]) > 1e38, np.inf, v[9])            # (or 0, where the gate is far below zero)
    assert np.array_equal(np.isnan(val(q)), ~np.isfinite(v)) and np.isnan(val(q)[[4]]).all() and np.isnan(val(q)[:, [7, 200]]).all()
    fine, e = np.isfinite(v), np.repeat(exps(s), 128, 1)
    plain = np.ones(T, dtype=bool)
    plain[[9]] = False
    A = np.abs(np.where(np.isnan(xv), 0, xv)) @ np.abs(np.where(np.isnan(wv), 0, wv)).T
    err = 2 * (7 * 2.0 ** -13 + 300 * 2.0 ** -24) * (np.abs(hg[:, inter:]) * 1.2 * A[:, :inter] + np.abs(hg[:, :inter]) * A[:, inter:]) + 2e-4 * np.abs(v)
    off = np.abs(val(q) * np.ldexp(1.0, e) - v)
    assert np.all((off <= 2.0 ** -4 * np.abs(v) + 2.0 ** -10 * np.ldexp(1.0, e) + err)[fine & plain[:, None]])
    assert np.all(exps(s)[4] == -126)
    clean = np.abs(np.where(fine, v, 0)).reshape(T, 2, 128).max(2)
    worst = np.where(fine, err, 0).reshape(T, 2, 128).max(2)
    most = np.ldexp(448.0, exps(s))
    assert np.all(((clean - worst <= most) & ((clean + worst > most / 2) | (exps(s) == -126)))[plain])


@pytest.mark.parametrize("T", [5, 300])
def test_gate_backward_of_what_is_not_finite(T):
    """Infinities and NaN in da, h and g are stored as NaN, and the block's scale is that of the others."""
    inter, inf, nan = 256, np.inf, np.nan
    rng = np.random.default_rng(4)
    da, hg = bf16(rng.standard_normal((T, inter))), bf16(rng.standard_normal((T, 2 * inter)))
    da[0, :3], hg[1, :3], hg[2, inter:inter + 3] = [inf, -inf, nan], [inf, -inf, nan], [inf, -inf, nan]
    da[3, :128] = nan
    hg[4, :4], hg[4, inter + 4] = [5e37, -5e37, 1e30, -1e30], 5e37
    da, hg = bf16(da), bf16(hg)
    q, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), dev(hg, BF16))
    with np.errstate(all="ignore"):
        value, slope = orc.gelu(hg[:, :inter])
        v = np.concatenate([da * (hg[:, inter:] * slope), da * value], 1)
    want, e = orc.store(v)
    assert np.array_equal(exps(s), e)
    assert np.array_equal(np.isnan(val(q)), np.isnan(want)) and np.isnan(want).sum() >= 3 * 5 + 128
    fine = ~np.isnan(want)
    off = np.abs(val(q) * np.ldexp(1.0, np.repeat(e, 128, 1)) - v)
    assert np.all((off <= 2.0 ** -4 * (1 + 1e-3) * np.abs(v) + 2.0 ** -10 * np.ldexp(1.0, np.repeat(e, 128, 1)))[fine])


# ---------------------------------------------------------------------------------------------------- every scale byte
def coded(q, b, rows=1):
    """8-bit rows with the given scale bytes: (values in 64 bits, q and s on the GPU)."""
    dq = torch.from_numpy(q.astype(np.float32)).to(E4M3)
    assert np.array_equal(val(dq), q, equal_nan=True)
    scale = np.where(b == 255, np.nan, np.ldexp(1.0, b.astype(int) - 127))
    values = q * np.repeat(np.repeat(scale, rows, 0), 128, 1)[:q.shape[0], :q.shape[1]]
    return values, dq.cuda(), torch.from_numpy(b.astype(np.uint8)).view(E8M0).cuda()


def codes_of(rng, *shape):
    return np.ldexp(8.0 + rng.integers(0, 8, shape), rng.integers(-2, 3, shape)) * rng.choice([-1.0, 1.0], shape)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("T,n_in,n_out", [(3, 384, 272), (70, 384, 784), (500, 384, 784), (2500, 384, 784), (12000, 384, 2064)])
def test_products_under_the_first_and_the_last_scale(T, n_in, n_out, dtype):
    """Scale byte 0 is 2^-127, 255 is NaN, also for codes that are 0; both apply to their block alone."""
    rng = np.random.default_rng(T)
    x, w = codes_of(rng, T, n_in), codes_of(rng, n_out, n_in)
    xb, wb = np.full((T, 3), 127), np.full((-(-n_out // 128), 3), 127)
    xb[1, :], wb[1, :] = 0, 247                                   # 2^-127 and 2^120: results of some 2^6
    xb[2, 1], x[2, 128:256], wb[2, 2], w[256:272, 256:] = 255, 0.0, 255, 0.0
    xb[0, :] = 60
    xv, xq, xs = coded(x, xb)
    wv, wq, ws = coded(w, wb, 128)
    got = mb.mb_linear_fp8_fwd(xq, xs, wq, ws, dtype=dtype).double().cpu().numpy()
    y, A = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    beyond = A > 1e38                                             # (row blocks under 2^127 with ordinary ones)
    nan = np.isnan(y)
    assert nan.any() and np.array_equal(np.isnan(got) & ~beyond, nan)
    fine = ~nan & ~beyond
    fast = dtype == BF16
    assert fine[1, 128:256].all()
    assert np.all(np.abs(got - y)[fine] <= ((n_in + 8) * 2.0 ** -24 * A + (7 * 2.0 ** -13 * A + 2.0 ** -8 * np.abs(y) if fast else 0) + 1e-37)[fine])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,n_in,n_out", [(5, 144, 80), (300, 1040, 400), (6000, 784, 528), (12000, 528, 528)])
def test_weight_gradient_under_the_first_and_the_last_scale(T, n_in, n_out, eight):
    rng = np.random.default_rng(T)
    x, xb = codes_of(rng, T, n_in), np.full((T, -(-n_in // 128)), 127)
    xb[1, 1], x[1, 128:], xb[0, 0] = 255, 0.0, 0
    xv, xq, xs = coded(x, xb)
    if eight:
        dyb = np.full((T, -(-n_out // 128)), 127)
        dyb[0, :] = 254 - 20
        dyv, dyq, dys = coded(codes_of(rng, T, n_out), dyb)
    else:
        dyv = bf16(rng.standard_normal((T, n_out)))
        dyv[0] *= 2.0 ** 107
        dyq, dys = dev(dyv, BF16), None
    xv[0, 128:] = 0.0
    xq.view(torch.uint8)[0, 128:] = 0
    got = mb.mb_linear_fp8_wgrad(dyq, xq, xs, dys=dys).double().cpu().numpy()
    want, A = dyv.T @ xv, np.abs(dyv).T @ np.abs(xv)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan) and nan[:, 128:min(256, n_in)].all() and not nan[:, :128].any()
    assert np.all(np.abs(got - want)[~nan] <= ((T + 40) * 2.0 ** -24 * A + 1e-37)[~nan])


def test_gate_under_the_first_and_the_last_scale():
    T, hidden, inter = 70, 256, 256
    rng = np.random.default_rng(8)
    x, w = codes_of(rng, T, hidden), codes_of(rng, 2 * inter, hidden)
    xb, wb = np.full((T, 2), 120), np.full((4, 2), 119)
    xb[1, 0], x[1, :128], wb[1, 1] = 255, 0.0, 255                # token 1; h of columns 128 ..
    xb[2, :], wb[0, :], wb[2, :] = 0, 240, 240
    x[3:] = 0.0
    x[0] = 0.0
    xv, xq, xs = coded(x, xb)
    wv, wq, ws = coded(w, wb, 128)
    q, s = mb.mb_geglu_fp8_act(xq, xs, wq, ws)
    hg, A = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    v = orc.gelu(hg[:, :inter])[0] * hg[:, inter:]
    assert np.array_equal(np.isnan(val(q)), np.isnan(v)) and np.isnan(v[1]).all() and np.isnan(v[:, 128:]).all() and np.isfinite(v[2, :128]).all()
    err = 2 * (7 * 2.0 ** -13 + 300 * 2.0 ** -24) * (np.abs(hg[:, inter:]) * 1.2 * A[:, :inter] + np.abs(hg[:, :inter]) * A[:, inter:]) + 2e-4 * np.abs(v)
    sc, fine = np.repeat(np.ldexp(1.0, exps(s)), 128, 1), np.isfinite(v)
    assert np.all((np.abs(val(q) * sc - v) <= 2.0 ** -4 * np.abs(v) + 2.0 ** -10 * sc + err)[fine])
    assert np.all(exps(s)[1] == -126) and np.all(exps(s)[:, 1] == -126)
    # backward: h | g in 8 bits
    hq, hb = codes_of(rng, T, 2 * inter), np.full((T, 4), 122)
    hb[1, 0], hq[1, :128], hb[2, 2], hb[4, 1] = 255, 0.0, 0, 255
    hv, hgq, hgs = coded(hq, hb)
    da = bf16(rng.standard_normal((T, inter)))
    da[2, :128] *= 2.0 ** 60
    da = bf16(da)
    q, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), hgq, hgs)
    value, slope = orc.gelu(hv[:, :inter])
    v = np.concatenate([da * (hv[:, inter:] * slope), da * value], 1)
    want, e = orc.store(v)
    assert np.array_equal(np.isnan(val(q)), np.isnan(want)) and np.isnan(want).sum() == 4 * 128
    assert np.array_equal(exps(s), e)
    sc, fine = np.repeat(np.ldexp(1.0, e), 128, 1), ~np.isnan(want)
    assert np.all((np.abs(val(q) * sc - v) <= 2.0 ** -4 * (1 + 1e-3) * np.abs(v) + 2.0 ** -10 * sc)[fine])


@pytest.mark.parametrize("eight", [False, True])
def test_gate_backward_decides_beside_a_border_in_64_bits(eight):
    """Blocks of one gradient each, da g GeLU'(h) within 1e-5 of 448 * 2^e: less than what 32 bits leave of many of them."""
    bits = 3 if eight else 7
    m = 1.0 + np.arange(2 ** bits) / 2.0 ** bits
    h = np.concatenate([-np.ldexp(m, k) for k in range(4)] + [np.ldexp(m, k) for k in (-1, 0)])
    h, a, g = (x.ravel() for x in np.meshgrid(h[h > -11], 1.0 + np.arange(128) / 128.0, m, indexing="ij"))
    v = np.abs(a * g * orc.gelu(h)[1])
    off = np.abs(v / np.ldexp(448.0, np.floor(np.log2(v / 448.0) + 0.5).astype(int)) - 1)
    pick = np.flatnonzero((off < (1e-4 if eight else 1e-5)) & (off > 1e-8))
    assert len(pick) >= (4 if eight else 100)
    da, hg = np.zeros((len(pick), 128)), np.zeros((len(pick), 256))
    at = np.arange(len(pick)) % 128                                # (by every lane and place in it)
    da[np.arange(len(pick)), at], hg[np.arange(len(pick)), at], hg[np.arange(len(pick)), 128 + at] = a[pick], h[pick], g[pick]
    if eight:
        hg, hgq, hgs = stored(hg)
    else:
        hgq, hgs = dev(hg, BF16), None
    _, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), hgq, hgs)
    value, slope = orc.gelu(hg[:, :128])
    want = orc.scale_exponents(np.concatenate([da * hg[:, 128:] * slope, da * value], 1))
    print(len(pick), "blocks,", (exps(s) != want).sum(0), "scales not the definition's")
    assert np.array_equal(exps(s)[:, 0], want[:, 0])


def test_act_of_sums_computed_too_small():
    """The other way round: h = 3 * 2^-8 is computed as some 2^-8.  What 64 bits find beyond the border takes a scale that holds it."""
    x, w = cancelling()
    w[:128, 8] = -0.02734375
    v, q, e, _, _ = act(x, w)
    ratio = q * np.repeat(np.ldexp(1.0, e), 128, 1) / v
    assert np.isfinite(q).all() and np.all((ratio >= (1 - 2.0 ** -4) / 3.1) & (ratio <= 1 + 2.0 ** -4))
    assert np.all(e <= orc.scale_exponents(v))


def test_gate_backward_decides_beside_the_slopes_zero():
    """Every bf16 h within 0.04 of it, da g GeLU'(h) within 1e-4 of 448 * 2^e."""
    h = -np.arange(0.7109375, 0.79296875, 2.0 ** -8)               # (the step of bf16 there)
    m = 1.0 + np.arange(128) / 128.0
    h, a, g = (x.ravel() for x in np.meshgrid(h, m, m, indexing="ij"))
    slope = orc.gelu(h)[1]
    v = np.abs(a * g * slope)
    off = np.abs(v / np.ldexp(448.0, np.floor(np.log2(v / 448.0) + 0.5).astype(int)) - 1)
    pick = np.flatnonzero((off < 1e-4) & (off > 1e-8 + 4e-10 * 0.5 / np.abs(slope)))
    assert len(pick) > 50 and len(np.unique(h[pick])) > 15
    da, hg = np.zeros((len(pick), 128)), np.zeros((len(pick), 256))
    at = np.arange(len(pick)) % 128
    da[np.arange(len(pick)), at], hg[np.arange(len(pick)), at], hg[np.arange(len(pick)), 128 + at] = a[pick], h[pick], g[pick]
    assert np.array_equal(bf16(hg), hg)
    _, s = mb.mb_gelu_gate_fp8_bwd(dev(da, BF16), dev(hg, BF16))
    assert np.array_equal(exps(s)[:, 0], orc.scale_exponents((da * hg[:, 128:] * orc.gelu(hg[:, :128])[1]))[:, 0])
