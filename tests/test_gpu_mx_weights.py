"""The bits that mxfp4 attention keeps of a probability, seen where the weighted rows cancel."""
import numpy as np
import pytest
import torch

from tests import _mx
from tests.test_gpu_mx_decode import _launch, _problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g", [1, 8, 16])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_cancelling_rows(D, g):
    """12 tokens of weight 1 whose values sum to 69 and 24 of weight p whose values sum to -137, p about 69 / 137 =
    0.50365: the output is (69 - 137 p) / (12 + 24 p), near zero, where bf16 is fine enough to show how p is
    rounded (its 9th to 16th bits are set and clear at random).

    Scores are exact (codes 0 and 1; products of q whose sum fits 24 bits).  A weight as two bf16 parts, each to
    the nearest, is off by 2^-8 2^-9 = 2^-17 of it; those of 1 are exact.  The exponent's argument (two
    products rounded, 2^-23 of a magnitude below 1) and the exponential (a unit, 2^-23) add 2^-22, the fp32 sums
    of 36 terms, the division and the last product 2^-24 of the sum of weighted magnitudes in each of their 8
    steps: 2^-20 covers them.  The result rounds to bf16, 2^-8 of it."""
    B, H, n = 64, 2, 36
    p = _problem(B, H, g, D, 16, 16, [n] * B, 3, [D, g], poison=False)
    rng = np.random.default_rng([D, g])
    k, v = np.zeros((len(p["kc"]), H, 16, D)), np.zeros((len(p["kc"]), H, 16, D))
    one = np.arange(n) % 3 == 0                                     # in every tile: each wave's maximum is theirs
    key, val = np.where(one, 0.0, 1.0), np.empty(n)
    val[one], val[~one] = [6.0] * 11 + [3.0], [-6.0] * 22 + [-4.0, -1.0]
    for i in range(B):
        for t in range(n):
            page = p["perm"][p["indptr"][i] + t // 16]
            k[page, :, t % 16, :3], v[page, :, t % 16] = key[t], val[t]
    p["kc"], p["vc"], p["scale"] = _mx.pack(k, "k"), _mx.pack(v, "v"), 1.0
    q = np.zeros((B, H * g, D))
    q[..., 0] = -0.68359375                                         # ln(69 / 137) + 0.00228..
    q[..., 1] = -0.0022852 + (rng.random((B, H * g)) - 0.5) * 2.0 ** -12
    q[..., 2] = rng.integers(0, 64, size=(B, H * g)) * 2.0 ** -22
    p["q"] = torch.from_numpy(q).to(torch.bfloat16)
    s = p["q"].double().numpy()[..., :3].sum(-1)
    assert (s.astype(np.float32) == s).all()
    w = np.exp(s)
    total = 12 + 24 * w
    ref, inexact, absv = (69 - 137 * w) / total, 137 * w / total, (69 + 137 * w) / total
    assert ((w > 0.5 + 2.0 ** -9) & (w < 0.5 + 2.0 ** -8)).all() and np.abs(ref).max() < 2.0 ** -9
    got = _launch(p)
    assert (got == got[..., :1]).all()
    err = np.abs(got[..., 0] - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -17 * inexact + 2.0 ** -20 * absv).all(), float((err / inexact).max() * 2 ** 17)


@pytest.mark.parametrize("g", [2, 16])
@pytest.mark.parametrize("top", [4.0, 7.5])
def test_the_largest_values(g, top):
    """Values of V at the type's largest, 6 2^125: no weight passes 1, so a dominant row does not leave fp32, also
    when its score lies above an earlier one by less than the running maximum's step of 2^8."""
    D, n = 128, 64
    p = _problem(3, 2, g, D, 64, 64, [n] * 3, 1, [g, int(top)], poison=False)
    k, v = np.zeros((len(p["kc"]), 2, 64, D)), np.zeros((len(p["kc"]), 2, 64, D))
    k[:, :, :, 0] = -6.0                                            # rows without weight: score -6 * 32
    k[:, :, 3, 0], k[:, :, 3, 1] = 0.0, 0.0                         # one early row, score 0
    k[:, :, 40, 0], k[:, :, 40, 1] = 0.0, 1.0                       # one later row, score top * ln 2
    v[:] = np.where(np.arange(D) % 2, -6.0, 6.0) * 2.0 ** 125
    p["kc"], p["vc"], p["scale"] = _mx.pack(k, "k"), _mx.pack(v, "v"), 1.0
    q = np.zeros((3, 2 * g, D))
    q[..., 0], q[..., 1] = 32.0, top * np.log(2)
    p["q"] = torch.from_numpy(q).to(torch.bfloat16)
    got = _launch(p)
    want = v[0, 0, 0]
    # every row has the same values: the weights' errors (2^-17), sums and division are far below bf16's 2^-8
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want)).all(), got[0, 0, :4]


@pytest.mark.parametrize("g", [2, 16])
def test_the_smallest_values(g):
    """Values of V at the type's smallest scale, 2^-120 to 6 2^-119: the weighted sums below fp32's normal range keep
    2^-149, 2^-20 of the smallest weight (2^-8) times the smallest value in each of the 40 rows."""
    D, n = 128, 40
    p = _problem(3, 2, g, D, 16, 16, [n] * 3, 3, [g, 3], poison=False)
    rng = np.random.default_rng(g)
    v = rng.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], size=(len(p["kc"]), 2, 16, D)) * 2.0 ** -119
    v[..., ::32] = 2.0 ** -119 * 6.0                                # every group's largest: its scale is 2^-119
    p["vc"] = _mx.pack(v, "v")
    assert np.array_equal(_mx.unpack(p["vc"], "v"), v)
    got, k = _launch(p), _mx.unpack(p["kc"], "k")
    q = p["q"].double().numpy()
    for i in range(3):
        pg, pos = p["perm"][p["indptr"][i] + np.arange(n) // 16], np.arange(n) % 16
        for h in range(2):
            ref, absv, qk = _mx.attend(q[i, h * g:(h + 1) * g], k[pg, h, pos], v[pg, h, pos], p["scale"])
            tol = _mx.attend_tolerance(ref * 2.0 ** 119, absv * 2.0 ** 119, qk, p["scale"], D, n) * 2.0 ** -119
            assert (np.abs(got[i, h * g:(h + 1) * g] - ref) <= tol + n * 2.0 ** -20 * absv).all()
