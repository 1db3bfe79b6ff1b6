"""The router and its gradient on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")

U = O.U32
# The weights: scores in float take an exponential (2 ulp of each of two), a tree sum of
# up to 512 (10 roundings) and a division; 32 half steps cover them, once for a score and
# once for the sum of the chosen ones.
W_TOL = 64 * U


def make_logits(T, E, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    l = rng.standard_normal((T, E)).astype(np.float32)
    if kind == "coarse":          # many equal logits
        l = np.round(l * 2) / 2
    elif kind == "flat":
        l[:] = 0.25
    elif kind == "wide":          # saturated sigmoids, softmax shares that underflow
        l *= 60
    elif kind == "masked":
        l[rng.random((T, E)) < 0.4] = -np.inf
        l[rng.random((T, E)) < 0.05] = np.nan
        l[T // 2] = -np.inf
        l[T - 1] = np.nan
        l[0] = np.finfo(np.float32).min
        if T > 3:
            l[3, :] = -np.inf
            l[3, E - 1] = 1.0
    elif kind == "inf":
        l[rng.random((T, E)) < 0.1] = np.inf
    return l


def run(l, k, bias=None, load=False, stream=None, **kw):
    T, E = l.shape
    c = L.make_route_cfg(T, E, k, **kw)
    lg = torch.from_numpy(l).cuda()
    b = None if bias is None else torch.from_numpy(np.asarray(bias, np.float32)).cuda()
    idx = torch.full((T, k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), float("nan"), device="cuda")
    ld = torch.full((E,), 5, dtype=torch.int32, device="cuda") if load else None
    L.moe_route(c, lg, b, idx, w, ld, stream=stream)
    torch.cuda.synchronize()
    return idx.cpu().numpy(), w.cpu().numpy(), None if ld is None else ld.cpu().numpy() - 5


def check(l, k, bias=None, **kw):
    idx, w, load = run(l, k, bias, load=True, **kw)
    ri, rw, rl = O.route(l, bias, k, **kw)
    bad = np.nonzero((idx != ri).any(1))[0]
    assert bad.size == 0, (bad[:5], idx[bad[:3]], ri[bad[:3]])
    # (weights that underflow in float are off by its smallest number at most)
    assert (np.abs(w - rw) <= W_TOL * np.abs(rw) + 1e-38).all(), np.abs(w - rw).max()
    assert np.array_equal(load, rl)


SHAPES = [(1, 1, 1), (1, 16, 2), (5, 2, 2), (64, 7, 3), (257, 64, 2), (130, 64, 8), (33, 65, 4), (100, 128, 1),
          (67, 200, 6), (129, 256, 8), (20, 500, 16), (19, 512, 16), (3, 16, 16)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_choices_and_weights(T, E, k, score, renorm):
    check(make_logits(T, E, T + E), k, score=score, renorm=renorm)
    bias = 0.1 * np.random.default_rng(1).standard_normal(E).astype(np.float32)
    check(make_logits(T, E, T + E + 1), k, bias, score=score, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,groups,top", [(16, 2, 4, 2), (256, 8, 8, 4), (64, 6, 8, 3), (60, 4, 5, 2), (24, 3, 24, 5),
                                            (512, 16, 2, 1), (36, 1, 12, 1), (8, 8, 2, 2), (500, 10, 125, 7),
                                            (160, 6, 8, 3), (192, 8, 4, 2)])
def test_groups(E, k, groups, top, score):
    kw = dict(score=score, groups=groups, top_groups=top)
    bias = 0.05 * np.random.default_rng(2).standard_normal(E).astype(np.float32)
    check(make_logits(83, E, E), k, bias, **kw)
    check(make_logits(83, E, E), k, None, renorm=0, **kw)
    check(make_logits(41, E, E, "masked"), k, bias, **kw)
    check(make_logits(41, E, E, "coarse"), k, None, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", ["coarse", "flat", "wide", "masked", "inf"])
@pytest.mark.parametrize("E,k", [(8, 2), (64, 8), (256, 8), (300, 16)])
def test_ties_masks_and_infinities(kind, E, k, score):
    l = make_logits(45, E, 9, kind)
    check(l, k, score=score)
    check(l, k, score=score, renorm=0)
    check(l, k, np.zeros(E, np.float32), score=score)                      # a fresh bias: ties stay ties
    check(l, k, np.arange(E, dtype=np.float32) % 3 * 0.125, score=score)   # equal values from unequal parts
    bias = 0.1 * np.random.default_rng(2).standard_normal(E).astype(np.float32)
    bias[1], bias[E // 2] = -np.inf, np.nan                                # two experts offline, one always taken
    bias[E - 1] = np.inf
    check(l, k, bias, score=score)


def test_scores_one_step_apart():
    """Neighbouring floats, whose sigmoids and biased scores differ by less than float resolves."""
    T, E = 64, 32
    rng = np.random.default_rng(0)
    base = np.float32(0.7) + np.zeros((T, E), np.float32)
    l = base + rng.integers(0, 4, (T, E)).astype(np.float32) * np.spacing(np.float32(0.7))
    for score in ("softmax", "sigmoid"):
        check(l, 4, score=score)
        check(l, 4, np.full(E, 0.3, np.float32), score=score)
        check(l, 4, np.full(E, 0.3, np.float32), score=score, groups=4, top_groups=2)


@pytest.mark.parametrize("E", [4, 5, 16, 60, 64, 128, 200, 512])
def test_single_live_expert_and_zeros(E):
    """One expert left (its logit 0, its value 0 and just beside it), wherever it stands."""
    l = np.full((E, E), -np.inf, np.float32)
    l[np.arange(E), np.arange(E)] = 0.0
    for score in ("softmax", "sigmoid"):
        check(l, min(E, 3), score=score)
        check(l, min(E, 3), np.full(E, -1.0 if score == "softmax" else -0.5, np.float32), score=score)   # values exactly 0
        if E % 4 == 0:
            check(l, 1, np.full(E, -0.5, np.float32), score=score, groups=E // 4 if E // 4 <= 16 else 4, top_groups=1)
    l = np.zeros((3, E), np.float32)
    l[1] = np.float32(1e-42) * np.arange(E)
    l[2] = -l[1]
    check(l, min(E, 4))


@pytest.mark.parametrize("T", [24576, 24577, 32771])
@pytest.mark.parametrize("E,k", [(64, 8), (37, 5)])
def test_many_tokens_of_up_to_64_experts(T, E, k):
    l = np.random.default_rng(T + E).standard_normal((T, E)).astype(np.float32)
    l[::1000, ::2] = -np.inf
    check(l, k, score="softmax")
    check(l, k, np.linspace(-0.1, 0.1, E).astype(np.float32), score="sigmoid")


def test_load_is_added_and_counts_every_choice():
    l = make_logits(4099, 48, 5)
    c = L.make_route_cfg(4099, 48, 4)
    lg = torch.from_numpy(l).cuda()
    idx, w = torch.empty(4099, 4, dtype=torch.int32, device="cuda"), torch.empty(4099, 4, device="cuda")
    load = torch.zeros(48, dtype=torch.int32, device="cuda")
    for _ in range(3):
        L.moe_route(c, lg, None, idx, w, load)
    assert torch.equal(load.cpu(), 3 * torch.bincount(idx.reshape(-1).cpu(), minlength=48).int())


def check_bwd(l, idx, dw, score, renorm, scale):
    T, E = l.shape
    k = idx.shape[1]
    c = L.make_route_cfg(T, E, k, score, renorm, scale=scale)
    w = O.route_weights(l, idx, score, renorm, scale).astype(np.float32)
    w[(idx < 0) | (idx >= E)] = np.nan          # takes no part
    dw = dw.astype(np.float32)
    ref, mag = O.route_bwd(l, idx, dw.astype(np.float64), score, renorm, scale)
    dl = torch.full((T, E), float("nan"), device="cuda")
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    L.moe_route_bwd(c, t(l), t(idx), t(w), t(dw), dl)
    got = dl.cpu().numpy()
    # a term is a product of up to four factors, each good to 64 half steps (W_TOL), summed over k <= 16 and E
    assert (np.abs(got - ref) <= 4 * W_TOL * mag + 1e-37).all(), np.max(np.abs(got - ref) / (mag + 1e-37))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("T,E,k", SHAPES + [(50, 6, 2), (70, 10, 3)])
def test_gradient(T, E, k, score, renorm):
    rng = np.random.default_rng(T * E)
    l = make_logits(T, E, T * E)
    idx = O.route(l, None, k, score, renorm)[0]
    check_bwd(l, idx, rng.standard_normal((T, k)), score, renorm, 1.0)
    l = make_logits(T, E, T * E, "masked")
    idx = O.route(l, None, k, score, renorm)[0]
    dw = rng.standard_normal((T, k))
    dw[idx < 0] = np.nan                        # nothing flows from a choice that is not there
    check_bwd(l, idx, dw, score, renorm, 2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [0, 1])
def test_gradient_of_foreign_and_repeated_choices(score, renorm):
    rng = np.random.default_rng(4)
    l = make_logits(40, 20, 4)
    idx = rng.integers(-2, 22, (40, 4)).astype(np.int32)
    idx[7] = 3                                  # the same expert four times
    idx[8] = -1
    check_bwd(l, idx, rng.standard_normal((40, 4)), score, renorm, 1.5)


def test_gradient_of_wide_logits():
    rng = np.random.default_rng(6)
    for score in ("softmax", "sigmoid"):
        for renorm in (0, 1):
            l = np.clip(make_logits(50, 24, 6) * 20, -60, 60)   # e^-60 and its square stay in float's range
            idx = O.route(l, None, 3, score, renorm)[0]
            check_bwd(l, idx, rng.standard_normal((50, 3)), score, renorm, 1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [0, 1])
def test_gradient_against_differences_of_the_router(score, renorm):
    """Central differences of moe_route itself, at logits whose choices do not change."""
    T, E, k, h = 30, 8, 2, 2.0 ** -6
    l = make_logits(T, E, 12)
    idx = O.route(l, None, k, score, renorm)[0]
    dw = np.random.default_rng(1).standard_normal((T, k)).astype(np.float32)
    ref, _ = O.route_bwd(l, idx, dw, score, renorm, 1.0)
    seen = 0
    for e in range(E):
        w = []
        for s in (h, -h):
            m = l.copy()
            m[:, e] += np.float32(s)
            i, v, _ = run(m, k, score=score, renorm=renorm)
            w.append((i, v.astype(np.float64)))
        same = (w[0][0] == idx).all(1) & (w[1][0] == idx).all(1)
        seen += same.sum()
        diff = ((w[0][1] - w[1][1]) * dw).sum(1) / (2 * h)
        # float rounding of two weights over 2 h, the shift's own rounding, and h^2 / 6 of third derivatives below 2
        tol = (2 * W_TOL / (2 * h) + h * h / 3 + 2.0 ** -22 / h) * np.abs(dw).sum(1) + 1e-7
        assert (np.abs(diff - ref[:, e])[same] <= tol[same]).all()
    assert seen > T * E / 2


def test_empty_batch_and_side_stream():
    c = L.make_route_cfg(0, 16, 2)
    z = torch.empty(0, device="cuda")
    load = torch.ones(16, dtype=torch.int32, device="cuda")
    L.moe_route(c, z, None, z.int(), z, load)
    L.moe_route_bwd(c, z, z.int(), z, z, z)
    assert (load == 1).all()
    l = make_logits(500, 64, 3)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    idx, w, _ = run(l, 4, stream=s)
    assert np.array_equal(idx, O.route(l, None, 4)[0])
