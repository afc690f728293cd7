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


def dense(c, o, lse):
    """Gradients in fp64 on the GPU, a (sequence, KV head) at a time: its packed rows are one matrix."""
    G, d = c.hq // c.hkv, c.d
    q, do, o = (x.double().view(-1, c.hkv, G, d) for x in (c.q, c.do, o))
    k, v, lse = c.k.double(), c.v.double(), lse.double().t().reshape(-1, c.hkv, G)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for s, n in enumerate(c.n):
        r, m = slice(int(c.cq[s]), int(c.cq[s + 1])), slice(int(c.ck[s]), int(c.ck[s]) + n)
        for g in range(c.hkv):
            Q, D, O, L, K, V = q[r, g].reshape(-1, d), do[r, g].reshape(-1, d), o[r, g].reshape(-1, d), lse[r, g].reshape(-1, 1), k[m, g], v[m, g]
            p = torch.exp(c.scale * (Q @ K.t()) - L)
            ds = p * (D @ V.t() - (D * O).sum(1, keepdim=True))
            dq[r, g] = (c.scale * (ds @ K)).view(-1, G, d)
            dk[m, g], dv[m, g] = c.scale * (ds.t() @ Q), p.t() @ D
    return dq.reshape(c.q.shape), dk, dv


@pytest.mark.parametrize("hq,hkv,d", [(9000, 3, 64), (20480, 1, 64), (4100, 2, 128)])
def test_more_heads_than_one_pass_over_statistics_holds(hq, hkv, d):
    """The backward's statistics go block by block of heads: groups that end inside a block, and more heads than their statistics fit
    the LDS for."""
    c = Case([3, 2], [400, 130], hq, hkv, d, seed=32)
    o, lse = c.fwd()
    for name, got, want in zip(("dq", "dk", "dv"), c.bwd(o, lse), dense(c, o, lse)):
        # one rounding of 2^-8 / sqrt(3) * 0.74, those to fp16 are an eighth of it; a quarter more (see cross_util)
        assert float((got.double() - want).norm() / want.norm()) < 1.25 * 0.74 * 2.0 ** -8 / 3 ** 0.5, name


def marked(c, kind):
    """nan in one query row (kind "q"), in all valid keys of a sequence ("all"), or in one run of 32 keys, a wave's turn in the form
    for few rows ("run"); O and LSE of the rows that see it are nan, all others as they were."""
    if kind == "q":
        c.q[int(c.cq[1]), 1] = float("nan")
        rows, heads = slice(int(c.cq[1]), int(c.cq[1]) + 1), slice(1, 2)
    else:
        a = int(c.ck[1])
        c.k[a:a + c.n[1], 0] = c.k[a:a + c.n[1], 0] if kind == "run" else float("nan")
        if kind == "run":
            c.k[a + 32:a + 64, 0] = float("nan")
        rows, heads = slice(int(c.cq[1]), int(c.cq[2])), slice(0, c.hq // c.hkv)
    hit = torch.zeros((c.Tq, c.hq), dtype=torch.bool, device="cuda")
    hit[rows, heads] = True
    return hit


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["q", "all", "run"])
@pytest.mark.parametrize("lq,kv", [([1, 2, 1], [70, 90, 5]), ([1, 2, 1], [3000, 2100, 5]), ([40, 30, 7], [70, 90, 5]), ([200, 300, 1], [3000, 2100, 5]),
                                   ([40, 3, 64], [2000, 3000, 77])])
def test_nan_stays_nan_and_where_it_is(lq, kv, kind, dtype):
    c = Case(lq, kv, 4, 2, 64, dtype, seed=33)
    o, lse = c.fwd()
    hit = marked(c, kind)
    o2, lse2 = c.fwd()
    assert torch.all(torch.isnan(o2[hit])) and torch.all(torch.isnan(lse2.t()[hit]))
    assert torch.equal(o2[~hit], o[~hit]) and torch.equal(lse2.t()[~hit], lse.t()[~hit])
