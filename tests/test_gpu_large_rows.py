"""Sorted rows and back where one thread for each piece of work would be more than a launch counts
(2^32 threads).  Whole numbers and powers of two: every result is exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")   # noqa: E731


def test_2_to_30_choices():
    """Dispatch, and the combine's backward over the rows that it wrote."""
    T, k, E, d = 1 << 26, 16, 512, 8
    R = T * k
    cfg = L.make_sorted_cfg(T, d, 8, E, k, "f32")
    assert L.moe_sorted_rows(cfg) == R and R // 16 * 64 >= 1 << 32
    idx = torch.randint(-3, E, (T, k), device="cuda", dtype=torch.int32)
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    x = torch.stack([(t % m).float() for m in (3, 5, 7, 11, 13, 17, 19, 23)], dim=1)
    rb, re, slot, src = i32(E), i32(E), i32(T, k), i32(R)
    rows = torch.full((R, d), -7.0, device="cuda")
    ws = torch.empty(L.moe_sorted_workspace_bytes(cfg, L.MOE_CALL_DISPATCH), dtype=torch.uint8, device="cuda")
    L.moe_sorted_dispatch(cfg, x, idx, rb, re, slot, src, rows, ws)
    flat = idx.view(-1)
    n = torch.stack([(flat == e).sum() for e in range(E)])
    live = int(n.sum())
    assert torch.equal(re.long(), n.cumsum(0)) and torch.equal(rb.long(), n.cumsum(0) - n)
    step = 1 << 24   # (rows that torch gathers at a time)
    for a in range(0, R, step):
        s = src[a:a + step + 1]
        if a >= live:
            assert bool((s == -1).all()) and bool((rows[a:a + step] == -7).all())
            continue
        s = s[:live - a]
        e = flat[s.long()]
        assert bool((e >= 0).all()) and bool(((e[1:] > e[:-1]) | ((e[1:] == e[:-1]) & (s[1:] > s[:-1]))).all()), a
        assert torch.equal(rows[a:min(a + step, live)], x[s[:step].long() // k]), a
    for a in range(0, T, 1 << 22):
        at, on = slot[a:a + (1 << 22)].reshape(-1), flat[a * k:(a + (1 << 22)) * k] >= 0
        i = torch.arange(a * k, a * k + at.numel(), device="cuda", dtype=torch.int32)
        assert bool((at[~on] == -1).all()) and torch.equal(src[at[on].long()], i[on]), a
    # backward of the combine: O is those rows
    w = 2.0 ** torch.randint(-3, 4, (T, k), device="cuda").float()
    w[idx < 0] = float("nan")
    dy = torch.stack([((t * m) % 9 - 4).float() for m in (1, 2, 4, 5, 7, 8, 1, 2)], dim=1)
    dO = torch.full_like(rows, -7.0)
    dw = torch.full((T, k), float("nan"), device="cuda")
    L.moe_sorted_combine_bwd(cfg, rows, slot, src, w, dy, dO, dw)
    want = (x * dy).sum(1, keepdim=True)
    for a in range(0, T, 1 << 22):
        q = slice(a, a + (1 << 22))
        assert torch.equal(dw[q], torch.where(idx[q] >= 0, want[q], 0.0)), a
    for a in range(0, live, step):
        s = src[a:min(a + step, live)].long()
        assert torch.equal(dO[a:a + s.numel()], w.view(-1)[s].unsqueeze(1) * dy[s // k]), a
    assert bool((dO[live:] == -7).all())
    del rows, dO, idx, slot, src, w, dw, flat, s, e
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_by_token_of_over_64_gib(dtype):
    """The combine, and the dispatch's gradient with the gate's part."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    T, d, E = ((1 << 24) if dtype == "bf16" else (1 << 23)) + 3, 2048, 4
    assert T * d * dt.itemsize // 16 > 1 << 32
    cfg = L.make_sorted_cfg(T, d, 64, E, 1, dtype)
    R = L.moe_sorted_rows(cfg)
    rows = torch.empty(R, d, device="cuda", dtype=dt)
    col = torch.arange(d, device="cuda") % 16
    row = lambda r: ((r % 13).unsqueeze(1) + col).to(dt)   # noqa: E731
    step = 1 << 20
    for a in range(0, R, step):
        rows[a:a + step] = row(torch.arange(a, min(a + step, R), device="cuda"))
    slot = torch.arange(T - 1, -1, -1, device="cuda", dtype=torch.int32).unsqueeze(1).contiguous()
    slot[::1001] = -1
    w = 2.0 ** torch.randint(-2, 3, (T, 1), device="cuda").float()
    Wg = torch.randint(-2, 3, (E, d), device="cuda").to(dt)
    dl = torch.randint(0, 2, (T, E), device="cuda").float()
    y = torch.full((T, d), -7.0, device="cuda", dtype=dt)
    for gate in (False, True):
        y.fill_(-7.0)
        if gate:
            L.moe_sorted_dispatch_bwd(cfg, slot, rows, y, Wg, dl)
        else:
            L.moe_sorted_combine(cfg, rows, slot, w, y)
        for a in range(0, T, step):
            s = slot[a:a + step]
            v = torch.where(s >= 0, row(s.squeeze(1)).float(), 0.0)
            v = v + dl[a:a + step] @ Wg.float() if gate else v * w[a:a + step]
            assert torch.equal(y[a:a + step], v.to(dt)), (gate, a)
    del rows, y
    torch.cuda.empty_cache()
