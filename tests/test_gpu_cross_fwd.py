"""Cross attention, forward, against the fp64 reference (tolerances: cross_util)."""
import numpy as np
import pytest
import torch

from paper_2412_07894_amd import binding
from cross_util import Case, check_fwd

pytestmark = pytest.mark.gpu

HEADS = [(1, 1), (2, 2), (6, 2), (8, 1), (20, 20), (10, 5), (40, 1), (16, 8)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_lengths(hq, hkv, d):
    """One token to several tiles on either side, empty ones on both."""
    lq = [1, 0, 31, 33, 64, 200, 257, 1, 5, 300, 17]
    kv = [1, 50, 63, 64, 65, 0, 129, 300, 31, 1, 32]
    c = Case(lq, kv, hq, hkv, d, seed=hq + d)
    check_fwd(c, *c.fwd(), what=f"{hq}/{hkv}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (8, 2), (32, 8), (16, 1), (30, 10)])
@pytest.mark.parametrize("lq", [[1] * 7, [1, 0, 2, 1, 0, 2, 2]])
def test_few_rows(lq, hq, hkv, d):
    """The form for few rows: keys in parts and turns, ends inside them, none at all."""
    if max(lq) * (hq // hkv) > 32:
        pytest.skip("not the form for few rows")
    c = Case(lq, [1, 31, 32, 0, 257, 2100, 5000], hq, hkv, d, seed=3)
    check_fwd(c, *c.fwd())
    c = Case(lq, [4096] * 7, hq, hkv, d, kv_lens=[0, 1, 33, 5000, -3, 4096, 2049], seed=4)
    check_fwd(c, *c.fwd())


@pytest.mark.parametrize("d", [64, 128])
def test_padded_and_outside_rows(d):
    """Padding and rows of no sequence hold nan and are not read; outputs of rows of no sequence stay as they were."""
    for lq in ([3, 40, 300, 7], [2, 1, 2, 2]):
        c = Case(lq, [130, 400, 70, 64], 4, 2, d, kv_lens=[100, 0, 900, 1], seed=5, front=13, back=9)
        o, lse = torch.full_like(c.q, 7.0), torch.full((4, c.Tq), 7.0, device="cuda")
        c.fwd(out=o, lse=lse)
        check_fwd(c, o, lse)
        off = torch.from_numpy(~c.q_rows).cuda()
        assert off.sum() == 22 and torch.all(o[off] == 7.0) and torch.all(lse[:, off] == 7.0)


@pytest.mark.parametrize("lq", [[1, 2, 2], [40, 100, 300]])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 1.0])
def test_scales(lq, scale):
    c = Case(lq, [100, 700, 1300], 4, 2, 128, scale=scale, seed=6)
    check_fwd(c, *c.fwd())


@pytest.mark.parametrize("lq", [[1, 2, 2], [40, 30, 60], [40, 100, 300]])
@pytest.mark.parametrize("size", [4.0, 16.0, 60.0])
def test_large_scores(lq, size):
    """Rows whose later keys exceed the first ones by far: the reference of a row has to follow (scores of standard deviation
    size^2: a row is one key in the end)."""
    c = Case(lq, [100, 700, 1300], 4, 2, 128, seed=7, size=size)
    for s, a in enumerate(c.ck[:-1]):
        c.k[int(a):int(a) + 64] *= 0.01
    check_fwd(c, *c.fwd())


@pytest.mark.parametrize("d", [64, 128])
def test_up_to_128_rows(d):
    """Tiles of 128 rows: own items whole and in parts, a list of them, scores that overflow a first guess, padded keys."""
    rng = np.random.default_rng(9)
    for hq, hkv, lq, kv, kw in ((2, 2, [128, 100, 33, 1, 0, 64], [130, 64, 0, 700, 5, 63], {}),
                                (9, 3, [42, 11, 1], [3000, 200, 1], {}),
                                (4, 4, [40, 128], [900, 2000], dict(kv_lens=[65, 1900], front=3, back=4)),
                                (4, 2, [60, 33, 64], [300, 900, 129], dict(size=40.0)),
                                (2, 2, rng.integers(0, 129, 700), rng.integers(0, 300, 700), {})):
        c = Case(lq, kv, hq, hkv, d, seed=19, **kw)
        assert 32 < c.max_q * hq // hkv <= 128
        check_fwd(c, *c.fwd(), f"{hq}/{hkv}")


def test_list_with_many_sequences():
    """More items than workgroups, several lists' worth of classes, striped and partitioned queues."""
    rng = np.random.default_rng(8)
    for hq, hkv, d in ((8, 8, 64), (6, 3, 128)):
        lq, kv = rng.integers(0, 90, 700), rng.integers(0, 120, 700)
        lq[5], kv[5], kv[9] = 1500, 900, 1700
        c = Case(lq, kv, hq, hkv, d, seed=9)
        check_fwd(c, *c.fwd())


@pytest.mark.parametrize("lq,kv", [([1], [6000]), ([2, 1], [3000, 70]), ([70], [4000]), ([64, 300], [2500, 0])])
def test_parts_give_way_to_a_small_workspace(lq, kv):
    """With the least workspace the keys stay whole: the same values up to the order of sums."""
    c = Case(lq, kv, 2, 1, 128, seed=10)
    o, lse = c.fwd()
    check_fwd(c, o, lse)
    need = 256 * 1024                          # enough for any list of these sizes, too little for parts of many rows
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    o2, lse2 = c.fwd(workspace=ws)
    check_fwd(c, o2, lse2)
    big = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")      # a workspace of a larger batch, dirty
    o3, lse3 = c.fwd(workspace=big)
    assert torch.equal(o, o3) and torch.equal(lse, lse3)


def test_bound_above_the_lengths():
    """Bounds far above the lengths change the form, not the values."""
    for lq in ([1, 2], [50, 300]):
        c = Case(lq, [100, 900], 2, 2, 64, seed=11, back=5000)
        c.max_q, c.max_kv = 4000, 5000
        check_fwd(c, *c.fwd())


@pytest.mark.parametrize("lq", [[1, 1, 2], [300, 40, 700]])
def test_graph_stream_and_repeats(lq):
    c = Case(lq, [500, 2000, 77], 4, 4, 64, seed=12)
    need = binding.cross_attn_workspace_bytes(c.Tq, c.Tk, 3, c.max_q, c.max_kv, 4, 4, 64, binding.HYD_BF16, False)
    ws, o, lse = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(c.q), torch.empty((4, c.Tq), device="cuda")
    run = lambda: c.fwd(workspace=ws, out=o, lse=lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(3):
        c.q.copy_(torch.randn(c.q.shape, device="cuda"))
        ref, ref_l = c.fwd()
        o.fill_(float("nan")); lse.fill_(float("nan")); ws.fill_(255 if rep == 1 else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref) and torch.equal(lse, ref_l), rep


@pytest.mark.parametrize("lq", [1, 70])
def test_offsets_past_32_bits(lq):
    """Key buffers beyond 4 GiB: 40 sequences of padded caches, 2^31 elements and more in front of the last one."""
    rows, hkv, d, n = 53000, 8, 128, 42
    k = torch.zeros((n * rows, hkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.randn((n * lq, 8, d), device="cuda").to(torch.bfloat16)
    cq = torch.arange(n + 1, dtype=torch.int32, device="cuda") * lq
    ck = torch.arange(n + 1, dtype=torch.int32, device="cuda") * rows
    lens = torch.full((n,), 300, dtype=torch.int32, device="cuda")
    for s in range(n):
        k[s * rows:s * rows + 300] = torch.randn((300, hkv, d), device="cuda").to(torch.bfloat16)
        v[s * rows:s * rows + 300] = torch.randn((300, hkv, d), device="cuda").to(torch.bfloat16)
    o, lse = binding.cross_attn_fwd(q, k, v, cq, ck, lq, 300, 0.1, kv_lens=lens)
    small = lambda x: torch.cat([x[s * rows:s * rows + 300] for s in range(n)])
    o2, lse2 = binding.cross_attn_fwd(q, small(k), small(v), cq, torch.arange(n + 1, dtype=torch.int32, device="cuda") * 300, lq, 300, 0.1)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2), (20, 20), (40, 1)])
def test_fp32_lengths(hq, hkv, d):
    lq = [1, 0, 31, 33, 64, 200, 257, 1, 5, 300, 17]
    kv = [1, 50, 63, 64, 65, 0, 129, 300, 31, 1, 32]
    c = Case(lq, kv, hq, hkv, d, "fp32", seed=hq + d)
    check_fwd(c, *c.fwd(), what=f"{hq}/{hkv}")


@pytest.mark.parametrize("lq", [[1, 2, 1, 1], [40, 100, 7, 260]])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 1.0])
def test_fp32_scales_padding_and_parts(lq, scale):
    c = Case(lq, [130, 2500, 70, 64], 4, 2, 128, "fp32", kv_lens=[100, 2400, 0, 900], scale=scale, seed=5, front=13, back=9)
    o, lse = torch.full_like(c.q, 7.0), torch.full((4, c.Tq), 7.0, device="cuda")
    c.fwd(out=o, lse=lse)
    check_fwd(c, o, lse)
    off = torch.from_numpy(~c.q_rows).cuda()
    assert torch.all(o[off] == 7.0) and torch.all(lse[:, off] == 7.0)
    ws = torch.empty(64 * 1024, dtype=torch.uint8, device="cuda")         # too little for parts
    check_fwd(c, *c.fwd(workspace=ws))


def test_fp32_list_with_many_sequences():
    rng = np.random.default_rng(8)
    lq, kv = rng.integers(0, 90, 300), rng.integers(0, 120, 300)
    lq[5], kv[5], kv[9] = 900, 600, 1100
    c = Case(lq, kv, 6, 3, 64, "fp32", seed=9)
    check_fwd(c, *c.fwd())
