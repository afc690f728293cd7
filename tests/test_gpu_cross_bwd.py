"""Cross attention, backward, against the fp64 reference of the same O and LSE (tolerances: cross_util), and against differences."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paper_2412_07894_amd import binding
from cross_util import Case, check_bwd, cu_of, np64

pytestmark = pytest.mark.gpu


def both(c, what="", **kw):
    o, lse = c.fwd()
    dq, dk, dv = c.bwd(o, lse, **kw)
    check_bwd(c, o, lse, dq, dk, dv, what)
    return o, lse, dq, dk, dv


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 2), (6, 2), (8, 1), (20, 20), (10, 5), (40, 1), (16, 8)])
def test_lengths(hq, hkv, d):
    lq = [1, 0, 31, 33, 64, 200, 257, 1, 5, 300, 17]
    kv = [1, 50, 63, 64, 65, 0, 129, 300, 31, 1, 32]
    both(Case(lq, kv, hq, hkv, d, seed=hq + d), f"{hq}/{hkv}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 2), (6, 2), (8, 1), (20, 20), (10, 5), (40, 1), (16, 8)])
def test_few_keys(hq, hkv, d):
    """At most 128 keys: the form that streams the rows once."""
    lq = [1, 0, 31, 33, 64, 200, 257, 1, 5, 300, 17, 700]
    kv = [1, 50, 63, 64, 65, 0, 128, 127, 31, 96, 32, 77]
    both(Case(lq, kv, hq, hkv, d, seed=hq + d), f"{hq}/{hkv}")


@pytest.mark.parametrize("d", [64, 128])
def test_few_keys_padded_in_parts_and_scaled(d):
    for scale, size in ((None, 1.0), (-0.2, 1e-6), (0.0, 1e4)):
        c = Case([3, 2000, 0, 7, 1500], [130, 400, 70, 64, 9], 4, 2, d, kv_lens=[100, 128, 900, 0, -4], scale=scale, seed=5, front=13, back=9)
        c.do *= size
        assert c.max_kv <= 128
        o, lse = c.fwd()
        outs = []
        for ws in (None, torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(255)):
            dq, dk, dv = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
            c.bwd(o, lse, dq=dq, dk=dk, dv=dv, workspace=ws)
            check_bwd(c, o, lse, dq, dk, dv)
            for x, on in ((dq, c.q_rows), (dk, c.kv_rows), (dv, c.kv_rows)):
                off = torch.from_numpy(~on).cuda()
                assert off.sum() == 22 and torch.all(x[off] == 7.0)
            outs.append((dq, dk, dv))
        assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("d", [64, 128])
def test_padded_and_outside_rows(d):
    """Padding and rows of no sequence hold nan and are not read; dK and dV are 0 in the padding, outputs of rows of no sequence
    stay as they were."""
    for lq in ([3, 40, 300, 7, 0], [2, 1, 2, 2, 1]):
        c = Case(lq, [130, 400, 70, 64, 9], 4, 2, d, kv_lens=[100, 0, 900, 1, -4], seed=5, front=13, back=9)
        o, lse = c.fwd()
        dq, dk, dv = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
        c.bwd(o, lse, dq=dq, dk=dk, dv=dv)
        check_bwd(c, o, lse, dq, dk, dv)
        for x, on in ((dq, c.q_rows), (dk, c.kv_rows), (dv, c.kv_rows)):
            off = torch.from_numpy(~on).cuda()
            assert off.sum() == 22 and torch.all(x[off] == 7.0)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.5])
def test_scales(scale):
    both(Case([40, 1, 300], [100, 700, 130], 4, 2, 128, scale=scale, seed=6))


@pytest.mark.parametrize("size", [1e-6, 1e-3, 1e4])
def test_scale_of_the_gradient(size):
    """dO of any size; powers of two are followed bit for bit."""
    c = Case([40, 1, 300], [100, 700, 130], 4, 2, 64, seed=7)
    c.do *= size
    o, lse, dq, dk, dv = both(c)
    c.do *= 2.0 ** -20
    for a, b in zip((dq, dk, dv), c.bwd(o, lse)):
        small = a.float().abs() > 2.0 ** -90                   # (no subnormal results)
        assert torch.equal((a.float() * 2.0 ** -20)[small], b.float()[small])


def test_few_keys_and_few_rows_in_parts():
    """Few items: dQ in parts of the keys, dK/dV in parts of the rows; with the least workspace they stay whole."""
    for lq, kv, hq, hkv in (([9, 30], [5000, 700], 2, 1), ([6000, 2500], [40, 77], 2, 2), ([900], [1500], 4, 1)):
        c = Case(lq, kv, hq, hkv, 128, seed=8)
        o, lse, dq, dk, dv = both(c)
        big = torch.full((512 << 20,), 255, dtype=torch.uint8, device="cuda")
        for a, b in zip((dq, dk, dv), c.bwd(o, lse, workspace=big)):
            assert torch.equal(a, b)
        full = binding.cross_attn_workspace_bytes(c.Tq, c.Tk, len(lq), c.max_q, c.max_kv, hq, hkv, 128, binding.HYD_BF16, True)
        rows = lambda most, r, size: min(16 * r, most) * 128 * size
        room = max(rows(65536, c.Tq * hq, 4), rows(131072, c.Tk * hkv, 8))
        small = torch.empty(full - (room + 255) // 256 * 256, dtype=torch.uint8, device="cuda")
        check_bwd(c, o, lse, *c.bwd(o, lse, workspace=small), what="least workspace")
        with pytest.raises(binding.HydError):
            c.bwd(o, lse, workspace=small[:-256])


def test_many_key_tiles_in_parts():
    """Two parts of 200 key tiles: more records of key tiles than CUs."""
    both(Case([1100], [200 * 256 - 5], 1, 1, 64, seed=28))


@pytest.mark.parametrize("d", [64, 128])
def test_few_items_in_parts_fp32(d):
    """The same in fp32, with padded keys and a sequence without any."""
    for lq, kv, hq, hkv, lens in (([9, 30, 2], [5000, 700, 40], 2, 1, [4777, 700, 0]), ([3000, 1, 2500], [30, 0, 70], 4, 2, [17, 0, 70])):
        c = Case(lq, kv, hq, hkv, d, kv_lens=lens, seed=18, dtype="fp32", front=3, back=2)
        o, lse = c.fwd()
        outs = []
        for fill in (0, 255):
            ws = torch.full((64 << 20,), fill, dtype=torch.uint8, device="cuda")
            dq, dk, dv = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
            c.bwd(o, lse, dq=dq, dk=dk, dv=dv, workspace=ws)
            check_bwd(c, o, lse, dq, dk, dv)
            for x, on in ((dq, c.q_rows), (dk, c.kv_rows), (dv, c.kv_rows)):
                assert torch.all(x[torch.from_numpy(~on).cuda()] == 7.0)
            outs.append((dq, dk, dv))
        assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("n,dtype", [(100, torch.bfloat16), (300, torch.bfloat16), (300, torch.float32)])
def test_offsets_past_32_bits(n, dtype):
    """2^31 elements and more in front of the last sequence, of queries (rows of no sequence) and of keys (a padded one)."""
    far, h, d, lq, scale = 2_200_000, 8, 128, [70, 200], 0.1
    rnd = lambda *shape: torch.randn(shape, device="cuda").to(dtype)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, do, k, v = rnd(270, h, d), rnd(270, h, d), rnd(2 * n, h, d), rnd(2 * n, h, d)
    cq, ck = i32(0, 70, 270), i32(0, n, 2 * n)
    o, lse = binding.cross_attn_fwd(q, k, v, cq, ck, 200, n, scale)
    want = binding.cross_attn_bwd(q, k, v, o, lse, do, cq, ck, 200, n, scale)

    # queries: all behind `far` rows of no sequence; keys: the first sequence's at 0, the last one's behind its padding
    Q, O, DO = (torch.cat([torch.empty((far, h, d), dtype=dtype, device="cuda"), x]) for x in (q, o, do))
    LSE = torch.cat([torch.empty((h, far), device="cuda"), lse], dim=1).contiguous()
    K, V = (torch.cat([x[:n], torch.empty((far - n, h, d), dtype=dtype, device="cuda"), x[n:]]) for x in (k, v))
    dq, dk, dv = (torch.full_like(x, 7.0) for x in (Q, K, V))
    binding.cross_attn_bwd(Q, K, V, O, LSE, DO, cq + far, i32(0, far, far + n), 200, n, scale, kv_lens=i32(n, n), dq=dq, dk=dk, dv=dv)
    assert torch.all(dq[:far] == 7.0)
    for x in (dk, dv):
        assert not x[n:far].any()
    # (the small call may take items in parts: sums in another order, rounded once)
    step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -14
    for a, b in zip((dq[far:], torch.cat([dk[:n], dk[far:]]), torch.cat([dv[:n], dv[far:]])), want):
        assert torch.all((a - b).abs() <= step * b.abs() + 2.0 ** -14 * b.abs().max())


@pytest.mark.parametrize("hq,hkv", [(64, 1), (192, 2), (128, 1), (300, 1)])
def test_many_heads_to_a_group(hq, hkv):
    """Groups of 64 to 300 heads: tokens of a quarter of a tile and of more than a tile, in the general form and with few keys."""
    for kv in ([50, 0, 128, 77], [50, 0, 300, 77]):
        both(Case([3, 5, 9, 40], kv, hq, hkv, 64, seed=hq), f"{hq}/{hkv}")
    both(Case([2, 5, 9], [50, 0, 130], hq, hkv, 64, "fp32", seed=hq), f"{hq}/{hkv}")


@pytest.mark.parametrize("longest", [1, 200])
def test_very_many_sequences(longest):
    """70000 sequences of one query and one key (one has more): O = V, dV = sum of the group's dO, dQ = dK = 0 there."""
    n = 70000
    kv = np.ones(n, dtype=np.int64)
    kv[n // 2] = longest
    ck = torch.from_numpy(cu_of(kv)).cuda()
    cq = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    rnd = lambda t, h: torch.randn((t, h, 64), device="cuda").to(torch.bfloat16)
    q, k, v, do = rnd(n, 2), rnd(int(kv.sum()), 1), rnd(int(kv.sum()), 1), rnd(n, 2)
    o, lse = binding.cross_attn_fwd(q, k, v, cq, ck, 1, longest, 0.125)
    dq, dk, dv = binding.cross_attn_bwd(q, k, v, o, lse, do, cq, ck, 1, longest, 0.125)
    one = torch.from_numpy(kv == 1).cuda()
    at = ck[:-1].long()[one]
    assert torch.equal(o[one], v[at].expand(-1, 2, -1))
    # scores of one key: LSE is the score, P = 1 within the score's error, 70 * 2^-24 * 0.125 |q| |k| < 1e-4
    want = do[one].float().sum(1, keepdim=True)
    size = do[one].float().abs().sum(1, keepdim=True)
    assert torch.all((dv[at].float() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 1e-4) * size)
    # dP - D: the same 64 products, summed in another order, times P, scale and a k or q of at most 6; in the general form P is an fp16
    # number and dP - D rounds to nothing above 64 * 2^-24 * sum |do v| < 64 * 2^-24 * 200
    assert dq[one].float().abs().max() <= 1e-3 and dk[at].float().abs().max() <= 2e-3


def test_list_with_many_sequences():
    rng = np.random.default_rng(8)
    for hq, hkv, d in ((8, 8, 64), (6, 3, 128)):
        lq, kv = rng.integers(0, 90, 700), rng.integers(0, 120, 700)
        lq[5], kv[5], kv[9] = 1500, 900, 1700
        both(Case(lq, kv, hq, hkv, d, seed=9))


def test_queries_or_keys_missing_altogether():
    """No token on one side: the other side's gradients are zeros."""
    c = Case([0, 0], [30, 300], 2, 2, 64, seed=10)
    c.max_q = 0
    dk, dv = torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
    c.bwd(c.q, torch.zeros((2, 0), device="cuda"), dk=dk, dv=dv)
    assert torch.all(dk == 0) and torch.all(dv == 0)
    c = Case([20, 300], [0, 0], 2, 2, 64, seed=10)
    o, lse = c.fwd()
    assert torch.all(o == 0) and torch.all(lse == -float("inf"))
    dq, _, _ = c.bwd(o, lse, dq=torch.full_like(c.q, 7.0))
    assert torch.all(dq == 0)


def test_differences():
    """The whole operator, forward and backward, against central differences of the fp64 forward along random directions."""
    c = Case([20, 70, 1], [50, 90, 33], 4, 2, 64, kv_lens=[50, 61, 33], seed=11)
    o, lse = c.fwd()
    grads = [np64(x) for x in c.bwd(o, lse)]
    q, k, v = c.cpu()
    do = np64(c.do)
    loss = lambda x: (co.fwd(*x, c.cq, c.ck, c.scale, c.kv_lens)[0] * do).sum()
    rng = np.random.default_rng(0)
    for which, g in enumerate(grads):
        for _ in range(3):
            t = rng.standard_normal(g.shape)
            up, down = [q, k, v], [q, k, v]
            up[which], down[which] = up[which] + 1e-5 * t, down[which] - 1e-5 * t
            slope = (loss(up) - loss(down)) / 2e-5
            # each element of the gradient is off by 2^-8 of itself and, through the O that is rounded to bf16, a little more; signs are
            # independent along a random direction: six standard deviations
            assert abs(slope - (g * t).sum()) <= 6 * 2 * 2.0 ** -8 * np.sqrt((g * t * g * t).sum()) + 1e-3, which


def test_graph_stream_and_repeats():
    c = Case([300, 40, 700, 1], [500, 2000, 77, 9], 4, 2, 64, seed=12)
    o, lse = c.fwd()
    need = binding.cross_attn_workspace_bytes(c.Tq, c.Tk, 4, c.max_q, c.max_kv, 4, 2, 64, binding.HYD_BF16, True)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.v)]
    run = lambda: c.bwd(o, lse, workspace=ws, dq=out[0], dk=out[1], dv=out[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(3):
        c.do.copy_(torch.randn(c.do.shape, device="cuda") * 10.0 ** rep)
        ref = c.bwd(o, lse)
        for x in out:
            x.fill_(float("nan"))
        ws.fill_(255 if rep == 1 else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), rep


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2), (20, 20), (40, 1)])
def test_fp32_lengths(hq, hkv, d):
    lq = [1, 0, 31, 33, 64, 200, 257, 1, 5, 300, 17]
    kv = [1, 50, 63, 64, 65, 0, 129, 300, 31, 1, 32]
    both(Case(lq, kv, hq, hkv, d, "fp32", seed=hq + d), f"{hq}/{hkv}")


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.5])
def test_fp32_scales_padding_and_outside_rows(scale):
    c = Case([3, 140, 300, 7, 0], [130, 400, 70, 64, 9], 4, 2, 128, "fp32", kv_lens=[100, 350, 0, 1, -4], scale=scale, seed=5, front=13, back=9)
    o, lse = c.fwd()
    dq, dk, dv = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
    c.bwd(o, lse, dq=dq, dk=dk, dv=dv)
    check_bwd(c, o, lse, dq, dk, dv)
    for x, on in ((dq, c.q_rows), (dk, c.kv_rows), (dv, c.kv_rows)):
        assert torch.all(x[torch.from_numpy(~on).cuda()] == 7.0)


def test_fp32_list_with_many_sequences_and_missing_sides():
    rng = np.random.default_rng(8)
    lq, kv = rng.integers(0, 90, 300), rng.integers(0, 120, 300)
    lq[5], kv[5], kv[9] = 900, 600, 1100
    both(Case(lq, kv, 6, 3, 64, "fp32", seed=9))
    c = Case([0, 0], [30, 300], 2, 2, 64, "fp32", seed=10)
    c.max_q = 0
    dk, dv = torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
    c.bwd(c.q, torch.zeros((2, 0), device="cuda"), dk=dk, dv=dv)
    assert torch.all(dk == 0) and torch.all(dv == 0)
    c = Case([20, 300], [0, 0], 2, 2, 64, "fp32", seed=10)
    o, lse = c.fwd()
    dq, _, _ = c.bwd(o, lse, dq=torch.full_like(c.q, 7.0))
    assert torch.all(o == 0) and torch.all(dq == 0)
