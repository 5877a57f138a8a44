"""Scales of the 8-bit results where they hang by a thread: sums that cancel, gates far below zero, slopes next to their zero."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc
from paper_2312_17482_amd import binding as mb
from tests.test_gpu_fp8 import BF16, bf16, dev, exps, stored, val

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
