"""Cross attention: values that only some rows hold stay with those rows."""
import pytest
import torch

from cross_util import Case, check_bwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [1e30, float("inf"), float("nan")])
@pytest.mark.parametrize("kv,lens", [([200, 0, 700], None), ([300, 300, 300], [200, 0, 257])])
def test_gradients_of_rows_without_keys_scale_nothing(kv, lens, value, d):
    """dO of a sequence without valid keys enters no result: dK and dV of the others are the same bits, whatever it holds, and dQ of
    its own rows is 0."""
    c = Case([40, 70, 300], kv, 4, 2, d, kv_lens=lens, seed=31)
    assert c.max_kv > 128 and c.n[1] == 0
    c.do *= 1e-6
    rows = slice(int(c.cq[1]), int(c.cq[2]))
    c.do[rows] = 0
    o, lse = c.fwd()
    want = c.bwd(o, lse)
    check_bwd(c, o, lse, *want)
    c.do[rows.start + 7, 1] = value
    got = c.bwd(o, lse)
    for name, a, b in zip(("dq", "dk", "dv"), got, want):
        assert torch.equal(a, b), name
