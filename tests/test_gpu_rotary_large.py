"""General rotary positions where a workgroup takes its most rows: from 65536 rows on sixteen of them, small heads and the widest."""
import math

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
