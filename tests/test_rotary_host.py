"""General rotary positions, host side: the frequency table against its formula, the reference against closed forms, and every
refusal (none of these calls launches anything)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from oracle import rope_oracle, rotary_oracle as ro
from paper_2412_07894_amd import binding

OK, NULL, SHAPE, DTYPE, HEADS, HEADDIM = range(6)
P = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2412_07894_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load()


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (24, 500000.0), (64, 10000.0), (128, 1e6), (1024, 10000.0)])
@pytest.mark.parametrize("kw", [{}, {"scaling": "linear", "factor": 8.0}, {"scaling": "linear", "factor": 0.5},
                                {"scaling": "parts", "factor": 4.0, "original_length": 4096.0},
                                {"scaling": "parts", "factor": 40.0, "original_length": 8192.0, "low": 0.0, "high": 4.0}])
def test_frequencies(lib, rot, base, kw):
    got = binding.rope_frequencies(rot, base, device="cpu", **kw)
    assert got.dtype == torch.float64 and got.numel() == rot // 2
    # exp and log of the reference are within a few units of 2^-52 of an exponent of at most log(1e6) = 14
    np.testing.assert_allclose(got.numpy(), ro.frequencies(rot, base, **kw), rtol=64 * 2.0 ** -52)


def test_frequencies_by_parts_ends(lib):
    """Fast pairs keep their frequency bit for bit, slow ones are interpolated."""
    plain = binding.rope_frequencies(128, 10000.0, device="cpu")
    parts = binding.rope_frequencies(128, 10000.0, "parts", 4.0, 8192.0, 1.0, 32.0, device="cpu")
    r = 8192.0 * plain / (2 * math.pi)
    assert torch.equal(parts[r > 32.001], plain[r > 32.001]) and (r > 32.001).any()
    assert torch.equal(parts[r < 0.999], plain[r < 0.999] / 4.0) and (r < 0.999).any()
    mid = (r > 1) & (r < 32)
    assert (parts[mid] < plain[mid]).all() and (parts[mid] > plain[mid] / 4).all()


def test_frequencies_refusals(lib):
    out = (ctypes.c_double * 512)()
    f = lambda rot=64, base=1e4, sc=2, factor=4.0, ol=4096.0, low=1.0, high=32.0, o=out: lib.hyd_rope_frequencies(rot, base, sc, factor, ol, low, high, o)
    assert f() == OK
    for rot in (0, -2, 3, 63, 1026):
        assert f(rot=rot) == HEADDIM
    for bad in (dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(sc=3), dict(sc=-1), dict(factor=0.0), dict(factor=float("nan")),
                dict(ol=0.0), dict(ol=float("inf")), dict(low=-1.0), dict(high=1.0), dict(high=float("nan"))):
        assert f(**bad) == SHAPE, bad
    assert f(sc=0, factor=0.0, ol=0.0) == OK and f(sc=1, ol=0.0) == OK      # what is not looked at may be anything
    assert f(o=None) == NULL
    with pytest.raises(ValueError):
        binding.rope_frequencies(64, scaling="cubic", device="cpu")
    with pytest.raises(binding.HydError):
        binding.rope_frequencies(7, device="cpu")


def call(lib, **kw):
    a = dict(q=P, hq=4, qs=512, qo=2 * P, qos=512, k=3 * P, hk=2, ks=256, ko=4 * P, kos=256, cu=P, starts=None, nseq=2, pos=None, T=16,
             d=128, fr=P, rot=128, layout=0, mag=1.0, inv=0, dt=0)
    a.update(kw)
    return lib.hyd_rope_rotate(a["q"], a["hq"], a["qs"], a["qo"], a["qos"], a["k"], a["hk"], a["ks"], a["ko"], a["kos"], a["cu"], a["starts"],
                               a["nseq"], a["pos"], a["T"], a["d"], a["fr"], a["rot"], a["layout"], a["mag"], a["inv"], a["dt"], None)


def test_rotate_refusals(lib):
    assert call(lib, dt=2) == DTYPE
    for bad in (dict(T=-1), dict(nseq=-1), dict(layout=2), dict(qs=511), dict(qos=0), dict(ks=255), dict(kos=255), dict(q=P + 1), dict(ko=P + 1),
                dict(dt=1, qs=512, q=P + 2), dict(qo=P, qos=1024), dict(ko=3 * P, kos=512)):
        assert call(lib, **bad) == SHAPE, bad
    for bad in (dict(hq=0), dict(hk=-1), dict(hq=8192, qs=1 << 20, qos=1 << 20)):
        assert call(lib, **bad) == HEADS, bad
    for bad in (dict(rot=0), dict(rot=127), dict(rot=130), dict(d=0, rot=2), dict(d=1026, rot=2, qs=1 << 20, qos=1 << 20)):
        assert call(lib, **bad) == HEADDIM, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(fr=None), dict(cu=None)):
        assert call(lib, **bad) == NULL, bad
    assert call(lib, T=0) == OK and call(lib, nseq=0) == OK


def test_binding_refusals():
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    fr = torch.zeros(32, dtype=torch.float64)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    for kw in (dict(), dict(cu_seqlens=cu, positions=cu), dict(positions=cu, starts=cu), dict(cu_seqlens=cu, layout="both"),
               dict(cu_seqlens=cu), dict(cu_seqlens=cu[:0]), dict(cu_seqlens=cu, k=q[:3]), dict(cu_seqlens=cu, k=q.float()),
               dict(cu_seqlens=cu, out=q[:, :1])):
        with pytest.raises(ValueError):
            binding.rope_rotate(q, fr, **kw)
    with pytest.raises(ValueError):
        binding.rope_rotate(q, fr.float(), cu_seqlens=cu)
    with pytest.raises(TypeError):
        binding.rope_rotate(q.half(), fr, cu_seqlens=cu)


def test_reference_closed_forms():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((9, 2, 64))
    fr = ro.frequencies(64, 10000.0)
    np.testing.assert_allclose(ro.rotate(x, ro.positions([0, 4, 4, 9], 9), fr), rope_oracle.rope_packed(x, [0, 4, 4, 9]), atol=1e-13)
    pos = list(range(100, 109))
    half = ro.rotate(x, pos, fr)
    perm = np.arange(64).reshape(2, 32).T.reshape(-1)          # half layout -> pairs side by side
    side = ro.rotate(x[..., perm], pos, fr, layout="interleaved")
    np.testing.assert_allclose(side, half[..., perm], atol=1e-13)
    back = ro.rotate(ro.rotate(x, pos, fr, magnitude=2.0), pos, fr, magnitude=0.5, inverse=True)
    np.testing.assert_allclose(back, x, atol=1e-13)
    y, g = rng.standard_normal(x.shape), None                  # <R x, y> = <x, R^T y>
    np.testing.assert_allclose((ro.rotate(x, pos, fr, magnitude=1.3) * y).sum(), (x * ro.rotate(y, pos, fr, magnitude=1.3, inverse=True)).sum(), rtol=1e-12)
    part = ro.rotate(x, pos, fr[:12])
    assert np.array_equal(part[..., 24:], x[..., 24:])
    assert ro.positions([1, 3], 5) == [None, 0, 1, None, None] and ro.positions([0, 2], 2, [7]) == [7, 8]
