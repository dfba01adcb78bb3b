"""Both weights of a gated product as halves of one fused tensor, whose widths let only one of them start on 16 bytes."""
import pytest
import torch

from gated_util import reference
from operator_util import DTYPES, assert_within, offsets_of
from test_gpu_gated_matmul import DEV, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_either_weight_off_16_bytes(dtype):
    """Many pieces of few rows, n = 4 mod 8: the path of rows that start anywhere is chosen whichever weight it is, so that the sums have the same order and bits."""
    from paper_2508_18376_amd import moe_gated_matmul
    G, k, n, dt = 64, 512, 516, DTYPES[dtype]
    off = offsets_of([1 + g % 2 for g in range(G)])
    x, w = make((int(off[-1]), k), dt, 1), make((G, k, 2 * n), dt, 2, k ** -0.5)
    results = []
    for ahead in (0, 4):  # values in front of the fused tensor
        place = torch.empty(ahead + w.numel(), dtype=dt, device=DEV)[ahead:].view(w.shape)
        place.copy_(w)
        w1, w3 = place[:, :, :n], place[:, :, n:]
        assert [t.data_ptr() % 16 for t in (w1, w3)] == ([0, 8] if ahead == 0 else [8, 0])
        h, saved = moe_gated_matmul(x.to(DEV), w1, w3, off.to(DEV), want_saved=True)
        results.append((h, saved))
    want = reference(x, w[:, :, :n], w[:, :, n:], off, "silu")
    for h, saved in results:
        assert_within(h, *want["h"], "h")
        assert_within(saved, *want["saved"], "saved")
    assert torch.equal(results[0][1], results[1][1]) and torch.equal(results[0][0], results[1][0])
