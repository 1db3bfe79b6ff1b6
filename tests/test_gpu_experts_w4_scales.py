"""4-bit weights under the smallest scale byte: 0 stands for 2^-127 like every byte but 255."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as O
from tests.test_gpu_experts_w4 import dev, laid_out, run

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def weights(d, f, byte, second, E=1):
    """Codes of every kind under one byte in the one matrix, ones on the diagonal in the other."""
    W, s = np.zeros((1, f, d // 2), np.uint8), np.full((1, f, d // 32), 127, np.uint8)
    V, v = np.zeros((1, d, f // 2), np.uint8), np.full((1, d, f // 32), 127, np.uint8)
    for i in range(32):
        (W if second else V)[0, i, i // 2] = 2 << (4 * (i % 2))
    (V if second else W)[0, :32, :16] = (np.arange(32)[:, None] + np.arange(16)) % 16 * 17
    (v if second else s)[:] = byte
    return [a.repeat(E, 0) for a in (W, s, V, v)]


# The three forms of the products: K split over a block's waves, blocks of 128 rows, laid out.
@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("T,d,f,E,dtype", [(1, 32, 32, 1, "f32"), (32, 32, 32, 1, "bf16"), (33, 64, 96, 3, "f32"),
                                           (80, 256, 1024, 48, "bf16"), (90, 160, 1056, 48, "f32"), (13000, 32, 1024, 1, "bf16")])
@pytest.mark.parametrize("byte", [0, 1])
def test_smallest_scale_bytes(T, d, f, E, dtype, second, byte):
    assert laid_out(T, d, f, E, dtype) == (T == 13000)
    W = weights(d, f, byte, second, E)
    x = torch.zeros(T, d)
    x[torch.arange(T), torch.arange(T) % 32] = 2.0 ** 100      # results far above the smallest numbers
    idx = (np.arange(T) % E).astype(np.int32)[:, None]
    y = run(x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda(), dev(idx), dev(np.ones((T, 1), np.float32)),
            [dev(a) for a in W], E, f, 1, dtype, "identity").double().cpu().numpy()
    A, B = O.w4_decode(W[0][:, :32], W[1][:, :32])[0], O.w4_decode(W[2][:, :32], W[3][:, :32])[0]
    want = x.double().numpy()[:, :32] @ A[:, :32].T @ B[:, :32].T
    assert np.array_equal(y[:, :32], want) and np.abs(want).max() == 6 * 2.0 ** (byte - 27)


def test_smallest_scale_byte_of_results_below_the_normal_numbers():
    """x = 1 at one input: y is that input's decoded weight, a multiple of 2^-128."""
    W = weights(32, 32, 0, False)
    x = torch.eye(32)
    y = run(x.cuda(), dev(np.zeros((32, 1), np.int32)), dev(np.ones((32, 1), np.float32)), [dev(a) for a in W], 1, 32, 1, "f32",
            "identity").double().cpu().numpy()
    assert np.array_equal(y, O.w4_decode(W[0], W[1])[0].T)
