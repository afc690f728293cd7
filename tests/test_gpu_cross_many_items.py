"""Cross attention with more (sequence, KV head) pairs than one launch can give a workgroup each: 2^24 of 256 threads, 2^23 of 512.
One query and one key to a sequence: O = V and LSE = the score; dV = the sum of the group's dO, dQ = dK = 0 up to roundings."""
import pytest
import torch

from paper_2412_07894_amd import binding

pytestmark = pytest.mark.gpu
HEADS, D = 512, 64


def data(n):
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    new = lambda: torch.randn((n, HEADS, D), generator=g, device="cuda", dtype=torch.bfloat16)
    return new, torch.arange(n + 1, dtype=torch.int32, device="cuda")


def test_forward_of_few_rows():
    n = 2 ** 24 // HEADS + 1
    new, cu = data(n)
    q, k, v = new(), new(), new()
    o, lse = binding.cross_attn_fwd(q, k, v, cu, cu, 1, 1, 0.125)
    assert torch.equal(o, v)
    for a in range(0, n, 4096):
        x, y = q[a:a + 4096].float(), k[a:a + 4096].float()
        score, size = (x * y).sum(-1) * 0.125, (x * y).abs().sum(-1) * 0.125
        # 64 products and sums on either side, the scale, its product with log2(e) and back: units of 2^-24
        assert torch.all((lse[:, a:a + 4096].t() - score).abs() <= (2 * 64 + 8) * 2.0 ** -24 * size)


def test_backward_of_few_keys():
    n = 2 ** 23 // HEADS + 1
    new, cu = data(n)
    q, k, v, do = new(), new(), new(), new()
    o, lse = binding.cross_attn_fwd(q, k, v, cu, cu, 1, 1, 0.125)
    dq, dk, dv = binding.cross_attn_bwd(q, k, v, o, lse, do, cu, cu, 1, 1, 0.125)
    # P = 1 within the score's error, below 1e-4, and its rounding to fp16; dV rounded once.  The fp16 copy of dO, brought to a largest
    # value in [1, 2) by a power of two, keeps 2^-25 of that unit where it is below fp16's normal range; the unit is at most max |dO|.
    size = do.float().abs()
    assert torch.all((dv.float() - do.float()).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2e-4) * size + 1.01 * 2.0 ** -25 * size.max())
    # dP - D: the same 64 products, summed in another order: below 2 * 64 * 2^-24 * sum |do v| < 2e-3 for sums up to 200, times P,
    # the scale and a k or q of at most 7
    assert dq.abs().max() <= 2e-3 and dk.abs().max() <= 2e-3
