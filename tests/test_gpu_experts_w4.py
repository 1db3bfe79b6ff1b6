"""The experts on 4-bit weights, and the quantiser, on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def weights(E, N, K, rng, spread=6):
    codes = rng.integers(0, 256, (E, N, K // 2), dtype=np.uint8)
    scales = rng.integers(118, 118 + spread, (E, N, K // 32), dtype=np.uint8)
    return codes, scales


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run(x, idx, w, W, E, f, k, dtype, act, ws=None, stream=None):
    T, d = x.shape
    c = L.make_w4_cfg(T, d, f, E, k, dtype, act)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if ws is None:
        ws = torch.full((max(16, L.moe_experts_w4_workspace_bytes(c)),), 255, dtype=torch.uint8, device="cuda")   # NaN everywhere
    y = torch.full((T, d), float("nan"), dtype=dt, device="cuda")
    L.moe_experts_w4(c, x, idx, w, *W, y, ws, stream=stream)
    torch.cuda.synchronize()
    return y


def inputs(T, d, f, E, k, dtype, seed, skew=None):
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(dt)
    if skew is None:
        idx = np.stack([rng.permutation(E)[:k] if E >= k else rng.integers(0, E, k) for _ in range(T)]).astype(np.int32)
    else:
        idx = rng.choice(E, (T, k), p=skew).astype(np.int32)   # the same expert may come twice
    w = rng.random((T, k)).astype(np.float32)
    W = [*weights(E, f, d, rng), *weights(E, d, f, rng)]
    return x, idx.reshape(T, k), w, W


def laid_out(n, d, f, E, dtype):
    return dtype == "bf16" and n >= 24 * E and n * d * f >= (3 << 27 if f >= 1024 else 1 << 30)


def check(y, x, idx, w, W, act, dtype):
    # act(W1 x) keeps 16 significant bits, or (many tokens) is rounded once to bfloat16
    part = 2.0 ** -8 if laid_out(idx.size, x.shape[1], W[0].shape[1], W[0].shape[0], dtype) else 2.0 ** -16
    ref, err = O.experts(x.double().numpy(), idx, w.astype(np.float64), O.w4_decode(W[0], W[1]), O.w4_decode(W[2], W[3]), act, part)
    got = y.double().cpu().numpy()
    tol = err + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (np.abs(ref) + err)   # y's own rounding
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), np.max(np.abs(got - ref) / (tol + 1e-300))


SHAPES = [  # T, d, f, E, k
    (1, 32, 32, 1, 1), (1, 128, 256, 4, 2), (1, 1024, 512, 16, 2), (2, 96, 160, 3, 1), (7, 736, 288, 24, 3),
    (16, 64, 96, 2, 2), (17, 64, 64, 1, 1), (33, 160, 128, 1, 1), (31, 224, 96, 8, 2), (32, 128, 128, 4, 2), (33, 128, 64, 4, 2),
    (64, 96, 64, 64, 1), (65, 96, 64, 1, 1), (21, 256, 64, 160, 6), (130, 64, 128, 3, 2), (200, 128, 96, 5, 4),
    (48, 512, 1056, 16, 2), (4, 64, 64, 512, 16), (9, 64, 32, 16, 16), (300, 32, 64, 512, 8), (513, 64, 96, 2, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,k", SHAPES)
def test_against_oracle(T, d, f, E, k, dtype):
    x, idx, w, W = inputs(T, d, f, E, k, dtype, T + d + E)
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, dtype, "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", dtype)


# Blocks of 128 rows in either product or both: tokens found by expert and by choice, in one
# wave, in a block and in the list; whole and part steps of 256 inputs, rows that end inside a
# block, K in one and several splits, more than 16 tokens an expert.
ROWS = [  # T, d, f, E, k
    (80, 256, 1024, 48, 2), (40, 160, 1056, 48, 2), (11, 384, 512, 160, 6), (7, 768, 1024, 64, 8), (150, 96, 4128, 8, 2),
    (90, 4128, 96, 8, 2), (600, 96, 160, 64, 2), (3, 2080, 1312, 16, 16), (24, 1024, 2048, 16, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,k", ROWS)
def test_blocks_of_rows(T, d, f, E, k, dtype):
    x, idx, w, W = inputs(T, d, f, E, k, dtype, T + d + E)
    idx[T // 2, 0] = -1
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, dtype, "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["identity", "relu", "gelu_erf"])
@pytest.mark.parametrize("T", [3, 70])
def test_activations(T, act, dtype):
    x, idx, w, W = inputs(T, 192, 320, 6, 2, dtype, 5)
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], 6, 320, 2, dtype, act)
    check(y, x, idx, w, W, act, dtype)


MANY = [  # T, d, f, E, k
    (24, 128, 128, 1, 1), (48, 128, 256, 2, 1), (47, 128, 128, 1, 1), (128, 256, 128, 1, 1), (129, 384, 128, 1, 1),
    (300, 128, 640, 3, 2), (257, 640, 128, 4, 2), (600, 128, 128, 16, 1), (512, 256, 384, 2, 2), (33, 128, 1152, 1, 1),
    (100, 128, 2048, 2, 2),
    # inputs, rows or both past whole 128s
    (64, 160, 128, 2, 2), (70, 128, 96, 2, 1), (300, 32, 32, 3, 2), (50, 96, 160, 2, 2), (64, 1056, 352, 2, 2),
    (130, 288, 1184, 2, 3), (340, 224, 416, 7, 1), (33, 416, 2080, 1, 1)]


@pytest.mark.parametrize("T,d,f,E,k", MANY)
def test_many_tokens(T, d, f, E, k):
    x, idx, w, W = inputs(T, d, f, E, k, "bf16", T + d + f)
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", "bf16")


# The laid-out products, where act(W1 x) is rounded once (half a step of bfloat16).
LAID = [(3200, 128, 1024, 3, 1), (1500, 128, 1152, 2, 2), (450, 1024, 1024, 1, 1), (127, 1536, 1024, 2, 3),
        (2050, 512, 640, 8, 2), (400, 2048, 1024, 16, 1), (24, 2048, 8320, 1, 1), (161, 1280, 2048, 1, 1),
        # inputs, rows or both past whole 128s
        (1030, 288, 1184, 2, 2), (420, 1056, 1056, 2, 1), (1024, 416, 2080, 7, 1), (200, 160, 6400, 1, 2),
        (2048, 512, 544, 8, 2), (64, 1056, 6016, 2, 1), (4100, 96, 1056, 2, 1), (13000, 32, 1024, 5, 1), (700, 1152, 2144, 24, 1)]


@pytest.mark.parametrize("T,d,f,E,k", LAID)
def test_many_tokens_laid_out(T, d, f, E, k):
    assert laid_out(T * k, d, f, E, "bf16")
    x, idx, w, W = inputs(T, d, f, E, k, "bf16", T + d + f)
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", "bf16")


@pytest.mark.parametrize("T,d,f", [(320, 128, 256), (1100, 128, 1024), (800, 160, 1184)])
@pytest.mark.parametrize("act", ["identity", "relu", "gelu_erf"])
def test_many_tokens_uneven(act, T, d, f):
    E, k = 6, 3
    x, idx, w, W = inputs(T, d, f, E, k, "bf16", 9, np.array([0.5, 0.0, 0.3, 0.15, 0.04, 0.01]))
    idx[::7, 1] = -1
    idx[T - 20:] = E
    w[(idx < 0) | (idx >= E)] = np.nan
    x[T - 20:] = float("inf")
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", act)
    x[T - 20:] = 0
    check(y, x, idx, np.nan_to_num(w), W, act, "bf16")
    again = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", act)
    assert torch.equal(y, again) and (y[T - 20:] == 0).all()


@pytest.mark.parametrize("T,d,f", [(60, 128, 128), (3200, 128, 1024), (420, 1056, 1056)])
def test_many_tokens_infinities_stay_with_their_token(T, d, f):
    E, k = 2, 1
    x, idx, w, W = inputs(T, d, f, E, k, "bf16", 1)
    ref = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", "relu")
    bad = x.clone()
    bad[3, 5], bad[8, 127] = float("inf"), float("nan")
    y = run(bad.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, "bf16", "relu")
    rest = [t for t in range(T) if t not in (3, 8)]
    assert torch.equal(y[rest], ref[rest]) and torch.isnan(y[8]).all() and not torch.isfinite(y[3]).any()


@pytest.mark.parametrize("d,f", [(160, 96), (160, 1056), (416, 1024), (96, 1184)])
def test_many_tokens_far_scales_at_the_rows_ends(d, f):
    """The last scale of a row NaN, or with codes of 0 the largest: no other row or token sees it."""
    T, E, k = 80 if f < 1024 else (3 << 27) // (d * f) + 1, 2, 1
    x, idx, w, W = inputs(T, d, f, E, k, "bf16", d)
    W[2][:, 5, -16:] = 0
    W[3][:, 5, -1] = 254
    W[0][:, f - 1, -16:] = 0
    W[1][:, f - 1, -1] = 254
    args = (x.cuda(), dev(idx), dev(w))
    y = run(*args, [dev(v) for v in W], E, f, k, "bf16", "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", "bf16")
    W[3][1, d - 1, -1] = 255
    bad = run(*args, [dev(v) for v in W], E, f, k, "bf16", "gelu_tanh")
    of = torch.from_numpy(idx[:, 0] == 1).cuda()
    assert torch.isnan(bad[of, d - 1]).all() and of.any()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[of, d - 1] = False
    assert torch.equal(bad[keep], y[keep])


@pytest.mark.parametrize("T", [10, 90, 400])
def test_skewed_and_repeated_choices(T):
    skew = np.array([0.9] + [0.1 / 7] * 7)
    x, idx, w, W = inputs(T, 64, 96, 8, 3, "bf16", T, skew)
    y = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], 8, 96, 3, "bf16", "gelu_tanh")
    check(y, x, idx, w, W, "gelu_tanh", "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 12, 150])
def test_padding_and_foreign_choices_take_no_part(T, dtype):
    E, k, f = 6, 3, 64
    x, idx, w, W = inputs(T, 64, f, E, k, dtype, T)
    idx[T - 1:] = -1                                 # a padding token: 0, whatever it holds
    idx[::4, 1] = E
    idx[::3, 0] = -2 ** 31
    idx[1::5, 2] = 2 ** 31 - 1
    w[(idx < 0) | (idx >= E)] = np.nan
    xd = x.clone()
    none = ((idx < 0) | (idx >= E)).all(1)
    xd[torch.from_numpy(none)] = float("inf")
    y = run(xd.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, dtype, "gelu_tanh")
    check(y, x, idx, np.nan_to_num(w), W, "gelu_tanh", dtype)
    assert (y[torch.from_numpy(none).cuda()] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_stay_with_their_token_and_column(dtype):
    T, E, k, d, f = 20, 2, 1, 96, 64
    x, idx, w, W = inputs(T, d, f, E, k, dtype, 1)
    ref = run(x.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, dtype, "relu")
    bad = x.clone()
    bad[3, 5], bad[8, 95], bad[11, 64] = float("inf"), float("nan"), float("-inf")
    y = run(bad.cuda(), dev(idx), dev(w), [dev(v) for v in W], E, f, k, dtype, "relu")
    rest = [t for t in range(T) if t not in (3, 8, 11)]
    assert torch.equal(y[rest], ref[rest]) and torch.isnan(y[8]).all() and not torch.isfinite(y[[3, 11]]).any()


def test_float_inputs_next_to_the_largest():
    """Parts are cut, not rounded: a float past the largest bfloat16 stays finite."""
    d, f = 32, 32
    x = torch.zeros(1, d)
    x[0, 4] = 3.4e38
    W1, s1 = np.zeros((1, f, d // 2), np.uint8), np.full((1, f, 1), 127 - 100, np.uint8)
    W1[0, :, 2] = 0x02                                # input 4: 1.0 * 2^-100
    W2, s2 = np.full((1, d, f // 2), 0x22, np.uint8), np.full((1, d, 1), 127, np.uint8)
    y = run(x.cuda(), dev(np.zeros((1, 1), np.int32)), dev(np.ones((1, 1), np.float32)), [dev(v) for v in (W1, s1, W2, s2)],
            1, f, 1, "f32", "identity")
    want = np.float64(np.float32(3.4e38)) * 2.0 ** -100 * 32
    assert np.abs(y.cpu().numpy() / want - 1).max() <= 40 * 2.0 ** -24


@pytest.mark.parametrize("byte", [1, 20, 126, 127, 128, 200, 240, 255])
def test_every_code_and_far_scales(byte):
    """x = 1 at one input: y is that input's decoded weight, through an identity W2."""
    d = f = 32
    codes = np.arange(16, dtype=np.uint8)
    W1 = np.zeros((1, f, d // 2), np.uint8)
    W1[0, :16, 0], W1[0, 16:, 0] = codes, codes << 4
    s1 = np.full((1, f, 1), byte, np.uint8)
    W2 = np.zeros((1, d, f // 2), np.uint8)
    for i in range(32):
        W2[0, i, i // 2] = 2 << (4 * (i % 2))
    s2 = np.full((1, d, 1), 127, np.uint8)
    for col in (0, 1):
        x = torch.zeros(1, d)
        x[0, col] = 1.0
        y = run(x.cuda(), dev(np.zeros((1, 1), np.int32)), dev(np.ones((1, 1), np.float32)), [dev(v) for v in (W1, s1, W2, s2)],
                1, f, 1, "f32", "identity")[0].cpu().numpy()
        want = O.w4_decode(W1, s1)[0, :, col]
        if byte == 255:
            assert np.isnan(y).all()
        else:
            assert np.array_equal(y.astype(np.float64), want), (y, want)


def test_same_bits_again_and_in_a_used_workspace():
    x, idx, w, W = inputs(90, 128, 160, 7, 3, "bf16", 2)
    a = [x.cuda(), dev(idx), dev(w), [dev(v) for v in W], 7, 160, 3, "bf16", "gelu_erf"]
    c = L.make_w4_cfg(200, 128, 160, 7, 3)
    ws = torch.zeros(L.moe_experts_w4_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    first = run(*a)
    for _ in range(4):
        assert torch.equal(run(*a, ws=ws), first)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert torch.equal(run(*a, ws=ws, stream=s), first)


def test_two_calls_at_once():
    """Two streams, a workspace each, the same weights; results as one after the other."""
    for T, d, f, E, k in ((6, 256, 512, 8, 2), (90, 128, 160, 7, 3), (200, 256, 384, 4, 2)):
        x, idx, w, W = inputs(T, d, f, E, k, "bf16", T)
        Wd = [dev(v) for v in W]
        sets = [(x.cuda(), dev(idx), dev(w)), (x.flip(0).contiguous().cuda(), dev(idx[::-1]), dev(w[::-1]))]
        want = [run(a, i, v, Wd, E, f, k, "bf16", "relu") for a, i, v in sets]
        c = L.make_w4_cfg(T, d, f, E, k, "bf16", "relu")
        ws = [torch.empty(L.moe_experts_w4_workspace_bytes(c), dtype=torch.uint8, device="cuda") for _ in sets]
        ys = [[torch.empty_like(v) for _ in range(8)] for v in want]
        streams = [torch.cuda.Stream() for _ in sets]
        torch.cuda.synchronize()
        for j in range(8):
            for (a, i, v), y, u, s in zip(sets, ys, ws, streams):
                L.moe_experts_w4(c, a, i, v, *Wd, y[j], u, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(y, r) for r, l in zip(want, ys) for y in l), T


@pytest.mark.parametrize("T,k", [(2 ** 21, 1), (2 ** 17, 16)])
def test_most_choices(T, k):
    """T * k = 2^21 in tiles of 16: more blocks down than a grid may have.  Token t is row t % 8 of x."""
    d = f = 32
    E = 2
    x, idx, w, W = inputs(8, d, f, E, k, "f32", 3, np.array([0.6, 0.4]))
    idx[5] = -1
    ref, err = O.experts(x.double().numpy(), idx, w.astype(np.float64), O.w4_decode(W[0], W[1]), O.w4_decode(W[2], W[3]), "relu", 2.0 ** -16)
    n = T // 8
    y = run(x.cuda().repeat(n, 1), dev(idx).repeat(n, 1), dev(w).repeat(n, 1), [dev(v) for v in W], E, f, k, "f32", "relu")
    y = y.view(n, 8, d)
    assert torch.equal(y, y[:1].expand_as(y))
    tol = err + 2.0 ** -24 * (np.abs(ref) + err)
    assert (np.abs(y[0].double().cpu().numpy() - ref) <= tol).all()


def test_empty_batch():
    W = [dev(v) for v in (*weights(2, 64, 32, np.random.default_rng(0)), *weights(2, 32, 64, np.random.default_rng(1)))]
    x = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda")
    i = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    L.moe_experts_w4(L.make_w4_cfg(0, 32, 64, 2, 2), x, i, i.float(), *W, x, None)
    torch.cuda.synchronize()


# ---------------------------------------------------------------------- quantiser
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantiser_codes(dtype):
    rng = np.random.default_rng(8)
    x = rng.standard_normal((37, 160)) * np.exp2(rng.integers(-140, 120, (37, 160 // 32)).repeat(32, 1))
    x[0, :8] = [7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]      # half way between codes
    x[0, 8:32] = 0
    x[1, :32] = 0
    x[2, 40], x[3, 100], x[4, 159] = np.inf, np.nan, -np.inf
    x[5, 32:64] = 3.3e38
    x[6, :32] = -0.0
    x[7, :32] = 1e-42
    x[8, :32] = 7 * 2.0 ** -3
    x[9, :32] = np.nextafter(np.float32(7 * 2.0 ** -3), np.float32(1))
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    c, s = L.alloc_w4(37, 160)
    L.moe_w4_quantize(t, c, s)
    rc, rs = O.w4_quantize(t.double().cpu().numpy())
    c, s = c.cpu().numpy(), s.cpu().numpy()
    assert np.array_equal(s, rs), (s != rs).nonzero()
    ok = np.repeat(rs != 255, 16, 1)
    assert np.array_equal(c[ok], rc[ok])


def test_quantised_layer_serves():
    """moe_w4_quantize's output is what moe_experts_w4 takes."""
    rng = np.random.default_rng(3)
    E, d, f, T, k = 3, 96, 128, 5, 2
    W1, W2 = (torch.from_numpy(0.02 * rng.standard_normal(s).astype(np.float32)).bfloat16().cuda() for s in ((E, f, d), (E, d, f)))
    q1, q2 = L.alloc_w4(E, f, d), L.alloc_w4(E, d, f)
    L.moe_w4_quantize(W1, *q1)
    L.moe_w4_quantize(W2, *q2)
    x, idx, w, _ = inputs(T, d, f, E, k, "bf16", 3)
    y = run(x.cuda(), dev(idx), dev(w), [*q1, *q2], E, f, k, "bf16", "gelu_tanh")
    check(y, x, idx, w, [v.cpu().numpy() for v in (*q1, *q2)], "gelu_tanh", "bf16")
