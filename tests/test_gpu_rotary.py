"""General rotary positions on the GPU against the fp64 reference.

bf16: an element may differ by half a step of the result plus the fp32 arithmetic before it.  fp32: the revolution is rounded to
fp32 below 1/2 (2^-26 of a revolution, 9.4e-8 in the angle), sine and cosine are good to 2 units of 2^-24 of 1 (1.2e-7) each,
their products with the magnitude, with the elements and the sum take three roundings of 2^-24 (1.8e-7): together below
4e-7 of magnitude * (|a| + |b|).  The copied elements have to be the same bits."""
import numpy as np
import pytest
import torch

from oracle import rotary_oracle as ro
from paper_2412_07894_amd import binding
import gpu_util as gu

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def data(T, h, d, dtype, seed, fused=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((T, h + fused, d), generator=g, device="cuda").to(DT[dtype])


def check(got, x, pos, freqs, dtype, rows=None, **kw):
    rows = list(range(x.shape[0])) if rows is None else rows
    xs, got = gu.to_np(x[rows]), gu.to_np(got[rows])
    pos = [pos[r] for r in rows]
    ref = ro.rotate(xs, pos, freqs, **kw)
    on = np.array([p is not None for p in pos])
    half, mag = len(freqs), abs(kw.get("magnitude", 1.0))
    size = np.abs(xs)
    pair = np.zeros_like(size)
    i, j = (np.arange(half), np.arange(half) + half) if kw.get("layout", "half") == "half" else (2 * np.arange(half), 2 * np.arange(half) + 1)
    pair[..., i] = pair[..., j] = size[..., i] + size[..., j]
    tol = 4e-7 * mag * pair
    if dtype == "bf16":
        tol = tol + gu.half_ulp_bf16(np.abs(ref) + tol) * (pair > 0)
    err = np.abs(got - ref)[on]
    assert np.all(np.isfinite(err)) and np.all(err <= tol[on]), float((err - tol[on]).max())
    assert np.array_equal(got[on][..., 2 * half:], xs[on][..., 2 * half:])


SHAPES = [([1], 1, 0, 64, 64), ([1, 7, 64, 0, 0, 184, 33], 3, 1, 128, 128), ([300, 5], 5, 5, 128, 64), ([17] * 70, 2, 1, 80, 24),
          ([40, 1, 90], 7, 1, 96, 42), ([2, 60], 2, 2, 256, 256), ([3], 2, 0, 2, 2), ([50], 3, 2, 66, 62), ([5, 6], 1, 1, 1024, 1000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("lengths,hq,hk,d,rot", SHAPES)
def test_rotate(lengths, hq, hk, d, rot, layout, dtype):
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    T = int(cu[-1])
    kw = dict(layout=layout, magnitude=1.0 if hk else 1.25, inverse=bool(hk))
    starts = np.arange(len(lengths)) * 1009
    fr = binding.rope_frequencies(rot, 10000.0, "parts", 4.0, 4096.0, device="cuda")
    q, k = data(T, hq, d, dtype, 1), data(T, hk, d, dtype, 2) if hk else None
    cud, std = torch.from_numpy(cu).cuda(), torch.from_numpy(starts.astype(np.int32)).cuda()
    got = binding.rope_rotate(q, fr, k=k, cu_seqlens=cud, starts=std, **kw)
    pos, frn = ro.positions(cu, T, starts), fr.cpu().numpy()
    y, z = got if hk else (got, None)
    check(y, q, pos, frn, dtype, **kw)
    if hk:
        check(z, k, pos, frn, dtype, **kw)
    # explicit positions and in place: the same bits
    w = q.clone()
    binding.rope_rotate(w, fr, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"), out=w, **kw)
    torch.cuda.synchronize()
    assert torch.equal(w, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [0, 1])
def test_parts_of_a_fused_projection(dtype, shift):
    """Q and K are views of one buffer, rotated in place; what lies beside them stays as it was.  shift: addresses that are
    multiples of an element only."""
    T, hq, hk, d, rot = 77, 4, 2, 64, 32
    row = (hq + 2 * hk) * d + 5 * shift
    buf = torch.randn((T * row + shift,), device="cuda").to(DT[dtype])
    before = buf.clone()
    view = lambda b, h0, h: torch.as_strided(b, (T, h, d), (row, d, 1), shift + h0 * d)
    q, k = view(buf, 0, hq), view(buf, hq, hk)
    fr = binding.rope_frequencies(rot, 10000.0, device="cuda")
    cu = torch.tensor([0, 30, T], dtype=torch.int32, device="cuda")
    binding.rope_rotate(q, fr, k=k, cu_seqlens=cu, out=q, k_out=k)
    pos, frn = ro.positions([0, 30, T], T), fr.cpu().numpy()
    check(q, view(before, 0, hq), pos, frn, dtype)
    check(k, view(before, hq, hk), pos, frn, dtype)
    keep = torch.ones_like(buf, dtype=torch.bool)
    view(keep, 0, hq + hk)[...] = False
    assert torch.equal(buf[keep], before[keep])


def test_rows_of_no_sequence_are_left():
    T, fr = 40, binding.rope_frequencies(64, device="cuda")
    q = data(T, 3, 64, "bf16", 5)
    out = torch.full_like(q, 7.0)
    cu = torch.tensor([4, 4, 20, 33], dtype=torch.int32, device="cuda")
    binding.rope_rotate(q, fr, cu_seqlens=cu, out=out)
    pos = ro.positions([4, 4, 20, 33], T)
    rows = [t for t in range(T) if pos[t] is not None]
    check(out, q, pos, fr.cpu().numpy(), "bf16", rows=rows)
    assert torch.all(out[:4] == 7.0) and torch.all(out[33:] == 7.0)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_many_sequences_and_far_positions(layout):
    """More sequences than one probe of 64 sees, empty ones among them, positions up to 2^30, negative ones too."""
    rng = np.random.default_rng(7)
    lengths = rng.integers(0, 9, 9000)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    T = int(cu[-1])
    starts = rng.integers(-1000, 1 << 30, len(lengths)).astype(np.int32)
    fr = binding.rope_frequencies(128, 10000.0, device="cuda")
    q = data(T, 2, 128, "fp32", 8)
    y = binding.rope_rotate(q, fr, cu_seqlens=torch.from_numpy(cu).cuda(), starts=torch.from_numpy(starts).cuda(), layout=layout)
    pos = ro.positions(cu, T, starts)
    rows = sorted(set(rng.integers(0, T, 400).tolist() + [0, T - 1]))
    # an angle of 2^30 radians is rounded to 2^-23 of one in the reference's own double arithmetic: 2^-23 of the pair on top
    xs, got = gu.to_np(q[rows]), gu.to_np(y[rows])
    ref = ro.rotate(xs, [pos[r] for r in rows], fr.cpu().numpy(), layout=layout)
    i, j = (np.arange(64), np.arange(64) + 64) if layout == "half" else (2 * np.arange(64), 2 * np.arange(64) + 1)
    pair = np.zeros_like(xs)
    pair[..., i] = pair[..., j] = np.abs(xs[..., i]) + np.abs(xs[..., j])
    assert np.all(np.abs(got - ref) <= (4e-7 + 2.0 ** -21) * pair)


def test_large_buffer_and_offsets_past_32_bits():
    """2^32 bytes and more between the first and the last row (strided rows of a larger buffer)."""
    T, d, stride = 33000, 128, 70000
    buf = torch.zeros((T * stride,), dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(buf, (T, 2, d), (stride, d, 1))
    q.copy_(data(T, 2, d, "bf16", 9))
    fr = binding.rope_frequencies(128, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    y = binding.rope_rotate(q, fr, cu_seqlens=cu)
    check(y, q, ro.positions([0, T], T), fr.cpu().numpy(), "bf16", rows=[0, 1, 16383, 30677, 30678, T - 2, T - 1])


def test_stream_graph_and_repeated_calls():
    """Captured into a graph and replayed with other values in the same buffers; equal calls give equal bits."""
    T, fr = 300, binding.rope_frequencies(64, 10000.0, "linear", 2.0, device="cuda")
    q, k = data(T, 4, 128, "bf16", 10), data(T, 1, 128, "bf16", 11)
    cu = torch.tensor([0, 100, T], dtype=torch.int32, device="cuda")
    out, k_out = torch.empty_like(q), torch.empty_like(k)
    run = lambda: binding.rope_rotate(q, fr, k=k, cu_seqlens=cu, out=out, k_out=k_out, layout="interleaved")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(3):
        q.copy_(data(T, 4, 128, "bf16", 20 + rep))
        ref, ref_k = binding.rope_rotate(q, fr, k=k, cu_seqlens=cu, layout="interleaved")
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(k_out, ref_k), rep
