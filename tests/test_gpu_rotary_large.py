"""General rotary positions where a workgroup takes its most rows: from 65536 rows on sixteen of them, small heads and the widest."""
import pytest
import torch

from paper_2412_07894_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def turned(x, pos, freqs, layout):
    """In fp64 on the GPU; also |a| + |b| of every element's pair."""
    x, half = x.double(), freqs.numel()
    ang = pos.double()[:, None, None] * freqs
    c, s = ang.cos(), ang.sin()
    i = torch.arange(half, device=x.device)
    i, j = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = x[..., i], x[..., j]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = a.abs() + b.abs()
    return y, size


def check(got, x, pos, freqs, layout, dtype):
    """The bounds of test_gpu_rotary, half a step of the result as 2^-8 of it; the fp64 angle itself is off by 2^-53 of at most
    2^28 radians, 2^-25."""
    y, size = turned(x, pos, freqs, layout)
    tol = (4e-7 + 2.0 ** -24) * size
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (y.abs() + tol) * (size > 0)
    assert torch.all((got.double() - y).abs() <= tol)


@pytest.mark.parametrize("heads,d,rot", [(1, 1024, 1024), (2, 1024, 1000), (3, 64, 64), (1, 64, 2)])
@pytest.mark.parametrize("layout,dtype", [("half", "bf16"), ("interleaved", "fp32")])
def test_many_rows(heads, d, rot, layout, dtype):
    T = 65536 + 5
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((T, heads, d), generator=g, device="cuda").to(DT[dtype])
    cu = torch.tensor([0, 1, 40000, T], dtype=torch.int32, device="cuda")
    freqs = binding.rope_frequencies(rot)
    y = binding.rope_rotate(x, freqs, cu_seqlens=cu, layout=layout)
    t = torch.arange(T, device="cuda")
    pos = t - cu[:-1].long()[(t[:, None] >= cu[1:].long()[None]).sum(1)]
    for a in range(0, T, 8192):
        check(y[a:a + 8192], x[a:a + 8192], pos[a:a + 8192], freqs, layout, dtype)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_more_rows_than_a_launch_has_threads_for(layout):
    """2^28 rows and more, sixteen to a workgroup of 256 threads: 2^32 threads."""
    T, first = 2 ** 28 + 37, 100_000_000
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x = torch.randn((T, 1, 2), generator=g, device="cuda", dtype=torch.bfloat16)
    cu = torch.tensor([0, first, T], dtype=torch.int32, device="cuda")
    freqs = binding.rope_frequencies(2)
    y = binding.rope_rotate(x, freqs, cu_seqlens=cu, layout=layout)
    step = 1 << 24
    for a in range(0, T, step):
        t = torch.arange(a, min(a + step, T), device="cuda")
        check(y[a:a + step], x[a:a + step], torch.where(t < first, t, t - first), freqs, layout, "bf16")


def test_second_row_of_workgroups():
    """2^22 workgroups of sixteen rows, and one row more: the grid gets its second row."""
    freqs = binding.rope_frequencies(2)
    for T in (2 ** 26, 2 ** 26 + 1):
        x = torch.randn((T, 1, 2), device="cuda", dtype=torch.bfloat16)
        pos = torch.arange(T, dtype=torch.int32, device="cuda")
        y = binding.rope_rotate(x, freqs, positions=pos)
        for a in range(0, T, 1 << 24):
            check(y[a:a + (1 << 24)], x[a:a + (1 << 24)], pos[a:a + (1 << 24)], freqs, "half", "bf16")
