"""The 8-bit checkpoint of values at the end of float's range."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def test_largest_floats_stay_finite():
    """Groups whose largest magnitude is one of the type's last values: 127 steps do not pass the range."""
    cfg = L.make_cfg(16, 64, 64, 1, 1, 16, 1, "f32", "identity")
    top = np.finfo(np.float32).max
    a = np.zeros((16, 64), np.float32)
    for r in range(16):                                       # row r: r steps of float below the largest
        a[r, 3], a[r, 40], a[r, 41] = top, -top, top / 4
        top = np.nextafter(top, np.float32(0))
    bufs = [torch.from_numpy(a.copy()).cuda() for _ in range(3)]
    end = torch.tensor([16], dtype=torch.int32, device="cuda")
    ck = L.alloc_ckpt(cfg)
    L.moe_ckpt_save(cfg, *bufs, None, end, ck)
    out = [torch.full_like(b, 7.0) for b in bufs]
    A = torch.full_like(bufs[0], 7.0)
    L.moe_ckpt_load(cfg, ck, None, end, out[0], out[1], A, out[2])
    for got in (*out, A):
        g = got.view(16, 64).double().cpu().numpy()
        assert np.isfinite(g).all()
        # 127 or 32 steps: the step is off by one of its last places at most, and half a one of the product
        assert (np.abs(g[:, [3, 40]] - a[:, [3, 40]]) <= 2.0 ** -22 * np.abs(a[:, [3, 40]])).all()
        assert (np.abs(g[:, 41] / a[:, 3] - 32 / 127) <= 2.0 ** -22).all()
        assert (np.delete(g, [3, 40, 41], 1) == 0).all()
