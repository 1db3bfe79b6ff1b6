"""The router at the ends of float's range, against the float64 oracle."""
import numpy as np
import pytest

from oracle import operators_oracle as O
from tests.test_gpu_router import check, check_bwd

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")

LOW = np.finfo(np.float32).min


def low_rows(E):
    """Rows whose live logits are all finite and at or below -1e30."""
    l = np.full((6, E), -np.inf, np.float32)
    l[0, E // 2] = LOW                                        # one expert left
    l[1, ::2] = -1e31
    l[2] = -1e31 * np.arange(1, E + 1, dtype=np.float32)      # apart: the first takes everything
    l[3] = LOW
    l[4, 1], l[4, E - 1] = -2e38, -3e38
    l[5, 0], l[5, E - 1] = np.nan, -1e30
    return l


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(4, 2), (16, 2), (64, 8), (200, 6), (512, 16)])
def test_live_logits_below_1e30(E, k, score, renorm):
    l = low_rows(E)
    kw = dict(score=score, renorm=renorm, scale=2.5)
    bias = 0.1 * np.random.default_rng(E).standard_normal(E).astype(np.float32)
    check(l, k, **kw)
    check(l, k, bias, **kw)
    check(l, k, np.linspace(-1, 0, E).astype(np.float32), **kw)
    if E % 16 == 0:
        check(l, k, bias, groups=4, top_groups=2, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [16, 64, 256])
def test_groups_of_far_biases(E, score):
    """Group values are sums: of two biases past 1e30 as of any others."""
    rng = np.random.default_rng(E)
    n = E // 4
    l = rng.standard_normal((32, E)).astype(np.float32)
    bias = 0.1 * rng.standard_normal(E).astype(np.float32)
    bias[0], bias[n], bias[n + 1] = 5e30, 2e30, 5e29          # 5e30 against 2.5e30
    for top in (1, 2):
        check(l, 2, bias, score=score, groups=4, top_groups=top)
    bias[[0, n]] = np.inf                                     # infinite sums tie: the lowest group
    bias[2], bias[n + 1] = -1.0, 5e29
    check(l, 2, bias, score=score, groups=4, top_groups=1)
    low = np.full(E, LOW, np.float32)                         # every group's second value is far below
    low[::n] = 0.0
    low[n], low[n + 1] = -2e30, -2e30                         # two of them are above one of the lowest
    for k in (1, 2):
        check(l, k, low, score=score, groups=4, top_groups=1)
        check(l, k, low, score=score, groups=4, top_groups=3)


@pytest.mark.parametrize("E,k", [(16, 2), (64, 8), (256, 8)])
def test_largest_scales_over_small_scores(E, k):
    """scale * s / sum is at most scale, whatever the sum is next to it."""
    l = np.full((8, E), -75.0, np.float32) - np.arange(8, dtype=np.float32)[:, None] / 4
    l += np.linspace(-1, 1, E).astype(np.float32)
    check(l, k, score="sigmoid", scale=1e7)
    check(l, k, score="sigmoid", scale=1e38)
    l[:, 0] = 0.0                                             # a softmax whose largest is not chosen
    bias = np.linspace(1, 2, E).astype(np.float32)
    bias[0] = -9.0
    check(l, k, bias, score="softmax", scale=1e7)
    check(l, k, bias, score="softmax", scale=1e38)


def test_large_scales_of_shares_that_underflow():
    """scale * s where s is below float's smallest numbers and the product is not."""
    E = 32
    l = np.zeros((40, E), np.float32)
    l[:, 1:] = -70.0 - 2.5 * np.arange(40, dtype=np.float32)[:, None] - np.arange(E - 1, dtype=np.float32) / 8
    for scale in (1.0, 1e10, 1e38):
        check(l, 4, score="softmax", renorm=0, scale=scale)
        check(l, 4, score="sigmoid", renorm=0, scale=scale)


@pytest.mark.parametrize("E", [4, 16, 40, 100, 200, 512])
def test_gradient_of_logits_below_2e38(E):
    """Shares of a plain softmax whose logits differ far below zero, or are all there."""
    l = low_rows(E)
    l[5, 1:E - 1] = -2.5e38
    k = 2
    idx = O.route(l, None, k, "softmax", 0)[0]
    idx[5] = [E - 1, 1]                                       # a choice with no share at all
    dw = np.random.default_rng(E).standard_normal((6, k))
    for score in ("softmax", "sigmoid"):
        for renorm in (0, 1):
            check_bwd(l, idx, dw, score, renorm, 1.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(16, 2), (64, 8), (512, 16)])
def test_gradient_of_the_largest_scale(E, k, score):
    """Renormalised weights of up to 1e38: their mean gradient is an ordinary number."""
    rng = np.random.default_rng(E)
    l = rng.standard_normal((20, E)).astype(np.float32)
    check_bwd(l, O.route(l, None, k, score, 1)[0], 10 + rng.random((20, k)), score, 1, 1e38)


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("E,k", [(16, 2), (64, 8), (256, 8)])
def test_weights_far_below_the_largest_logit(E, k, renorm):
    """Shares of e^-70: the difference to the largest logit is no float, and its rounding not the weight's."""
    rng = np.random.default_rng(E)
    l = (-35 + rng.standard_normal((200, E))).astype(np.float32)
    l[:, 0] = 35 + rng.random(200)                            # the largest, which the bias keeps out
    bias = np.linspace(1, 2, E).astype(np.float32)
    bias[0] = -9.0
    check(l, k, bias, score="softmax", renorm=renorm)
