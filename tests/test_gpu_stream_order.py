"""Layer steps on a stream that is not the current one, given as an object or as a handle, with the weight
gradients on a second one: the bits of the step on one stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")

T, D, F, E, K = 4000, 256, 512, 8, 2
NAMES = ("y", "dx", "dW1", "dW2", "dWg")


def _step(sorted_rows, seed):
    torch.manual_seed(seed)
    rn = lambda *s, std=1.0: (torch.randn(*s, device="cuda") * std).bfloat16()   # noqa: E731
    x, Wg, W1, W2, dy = rn(T, D), rn(E, D, std=0.05), rn(E, F, D, std=0.05), rn(E, D, F, std=0.05), rn(T, D)
    if sorted_rows:
        b = L.alloc_sorted(L.make_sorted_cfg(T, D, F, E, K))
        fwd, bwd = L.sorted_layer_forward, L.sorted_layer_backward
    else:
        b = L.alloc_layer(L.make_cfg(T, D, F, E, K, L.moe_capacity(T, E, K, 5, 4)))
        fwd, bwd = L.layer_forward, L.layer_backward

    def run(stream, dw_stream):
        for n in NAMES + ("dO", "dH"):
            getattr(b, n).fill_(3.0)          # (what a product that does not wait would read)
        torch.cuda.synchronize()
        fwd(b, x, Wg, None, W1, W2, stream)
        bwd(b, x, Wg, dy, stream, dw_stream)
        torch.cuda.synchronize()
        return {n: getattr(b, n).clone() for n in NAMES}
    return run


@pytest.mark.parametrize("chain", ["object", "handle", "current", "null handle"])
@pytest.mark.parametrize("dw", ["object", "handle"])
@pytest.mark.parametrize("sorted_rows", [False, True])
def test_step_on_two_streams(sorted_rows, dw, chain):
    run = _step(sorted_rows, 5)
    want = run(None, None)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    stream = {"object": main, "handle": main.cuda_stream, "current": None, "null handle": 0}[chain]
    for _ in range(3):
        got = run(stream, side if dw == "object" else side.cuda_stream)
        for n in NAMES:
            assert torch.equal(got[n], want[n]), n
