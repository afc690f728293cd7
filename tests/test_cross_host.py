"""Cross attention, host side: sizes of the workspace and every refusal (none of these calls launches anything), and the reference
against closed forms and differences."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import attn_oracle, cross_oracle as co
from paper_2412_07894_amd import binding

OK, NULL, SHAPE, DTYPE, HEADS, HEADDIM, SEQLENS, WORKSPACE = range(8)
P = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2412_07894_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load()


def host(vals):
    arr = (ctypes.c_int32 * len(vals))(*vals)
    return arr, ctypes.cast(arr, ctypes.c_void_p)


def fwd(lib, **kw):
    a = dict(q=P, k=P, v=P, cq=P, ck=P, kl=None, nseq=2, cqh=None, ckh=None, Tq=100, Tk=300, mq=60, mk=200, hq=4, hkv=2, d=128, scale=0.1, dt=0,
             o=P, lse=P, ws=P, wb=1 << 30)
    a.update(kw)
    return lib.hyd_cross_attn_fwd(a["q"], a["k"], a["v"], a["cq"], a["ck"], a["kl"], a["nseq"], a["cqh"], a["ckh"], a["Tq"], a["Tk"], a["mq"],
                                  a["mk"], a["hq"], a["hkv"], a["d"], a["scale"], a["dt"], a["o"], a["lse"], a["ws"], a["wb"], None)


COMMON = [(dict(dt=2), DTYPE), (dict(Tq=-1), SHAPE), (dict(Tk=-1), SHAPE), (dict(nseq=-1), SHAPE), (dict(nseq=0), SHAPE), (dict(mq=-1), SHAPE),
          (dict(mk=-1), SHAPE), (dict(mq=101), SHAPE), (dict(mk=301), SHAPE), (dict(mq=0), SHAPE), (dict(hq=0), HEADS), (dict(hkv=0), HEADS),
          (dict(hq=5), HEADS), (dict(d=96), HEADDIM), (dict(d=256), HEADDIM), (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL),
          (dict(cq=None), NULL), (dict(ck=None), NULL), (dict(ws=None), WORKSPACE), (dict(ws=P + 64), WORKSPACE), (dict(wb=100), WORKSPACE),
          (dict(Tk=1 << 23, mk=1 << 22), SHAPE),               # 2^22 * 2 * 128 * 2 = 2^31 bytes of keys
          (dict(Tq=1 << 22, mq=1 << 21), SHAPE),               # 2^21 * 4 * 128 * 2 = 2^31 bytes of queries
          (dict(q=P + 2), SHAPE), (dict(k=P + 8), SHAPE), (dict(v=P + 4), SHAPE),                     # rows move 16 bytes at a time
          (dict(Tq=1 << 30, mq=1), SHAPE),                     # 2^31 packed rows
          (dict(Tq=10, mq=1, hq=1 << 16, hkv=1 << 16), SHAPE)]  # a tile of queries beyond a buffer resource
SEQ = [([0, 70, 100], None, SHAPE), ([-1, 60, 100], None, SEQLENS), ([0, 60, 101], None, SEQLENS), ([0, 60, 50], None, SEQLENS),
       (None, [0, 201, 300], SHAPE), (None, [-1, 100, 300], SEQLENS), (None, [0, 100, 301], SEQLENS), (None, [0, 200, 190], SEQLENS)]


@pytest.mark.parametrize("kw,code", COMMON + [(dict(o=None), NULL), (dict(lse=None), NULL)])
def test_forward_refusals(lib, kw, code):
    assert fwd(lib, **kw) == code


@pytest.mark.parametrize("cq,ck,code", SEQ)
def test_forward_host_lengths(lib, cq, ck, code):
    keep, p = host(cq or ck)
    assert fwd(lib, **{"cqh" if cq else "ckh": p}) == code


def bwd(lib, **kw):
    a = dict(q=P, k=P, v=P, o=P, lse=P, do=P, cq=P, ck=P, kl=None, nseq=2, cqh=None, ckh=None, Tq=100, Tk=300, mq=60, mk=200, hq=4, hkv=2, d=128,
             scale=0.1, dt=0, dq=P, dk=P, dv=P, ws=P, wb=1 << 32)
    a.update(kw)
    return lib.hyd_cross_attn_bwd(a["q"], a["k"], a["v"], a["o"], a["lse"], a["do"], a["cq"], a["ck"], a["kl"], a["nseq"], a["cqh"], a["ckh"],
                                  a["Tq"], a["Tk"], a["mq"], a["mk"], a["hq"], a["hkv"], a["d"], a["scale"], a["dt"], a["dq"], a["dk"], a["dv"],
                                  a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,code", COMMON + [(dict([(n, None)]), NULL) for n in ("o", "lse", "do", "dq", "dk", "dv")])
def test_backward_refusals(lib, kw, code):
    assert bwd(lib, **kw) == code


@pytest.mark.parametrize("cq,ck,code", SEQ)
def test_backward_host_lengths(lib, cq, ck, code):
    keep, p = host(cq or ck)
    assert bwd(lib, **{"cqh" if cq else "ckh": p}) == code


def test_nothing_to_do(lib):
    assert bwd(lib, Tq=0, mq=0, Tk=0, mk=0) == OK and bwd(lib, Tq=0, mq=0, Tk=0, mk=0, nseq=0, ws=None) == OK
    assert fwd(lib, Tq=0, mq=0) == OK and fwd(lib, Tq=0, mq=0, nseq=0) == OK
    assert fwd(lib, Tq=0, mq=0, q=None, o=None, ws=None, wb=0) == OK


def test_workspace_never_falls():
    rng = np.random.default_rng(0)
    for is_bwd in (0, 1):
        for dt in (binding.HYD_BF16, binding.HYD_FP32):
            for _ in range(300):
                hkv = int(rng.choice([1, 2, 8, 20]))
                hq, d = hkv * int(rng.choice([1, 4, 5])), int(rng.choice([64, 128]))
                a = [int(2 ** rng.uniform(0, 15)) for _ in range(5)]
                a[3], a[4] = min(a[3], a[0]), min(a[4], a[1])
                b = [x + int(rng.integers(0, 3000)) * int(rng.integers(0, 2)) for x in a]
                b[3], b[4] = min(b[3], b[0]), min(b[4], b[1])
                sa, sb = (binding.cross_attn_workspace_bytes(*x, hq, hkv, d, dt, is_bwd) for x in (a, b))
                assert 0 < sa <= sb and sa % 256 == 0, (a, b)
    assert binding.cross_attn_workspace_bytes(10, 10, 1, 11, 10, 1, 1, 64, 0, 0) == 0
    assert binding.cross_attn_workspace_bytes(10, 10, 1, 10, 10, 3, 2, 64, 0, 0) == 0


def test_binding_refusals():
    q, k = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((6, 1, 64), dtype=torch.bfloat16)
    cq, ck = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([0, 6], dtype=torch.int32)
    for a in ((q[0], k, k, cq, ck), (q, k.float(), k, cq, ck), (q, k, k[:5], cq, ck), (q, k, k, cq, ck[:1]), (q, k, k, cq.long(), ck),
              (q.transpose(0, 1), k, k, cq, ck), (q, k, k, cq[:0], ck[:0]), (q, k, k, cq, ck)):          # the last: not on a GPU
        with pytest.raises(ValueError):
            binding.cross_attn_fwd(*a, 4, 6, 0.1)
    with pytest.raises(ValueError):
        binding.cross_attn_fwd(q, k, k, cq, ck, 4, 6, 0.1, out=q[:3])
    with pytest.raises(ValueError):
        binding.cross_attn_fwd(q, k, k, cq, ck, 4, 6, 0.1, cu_q_host=[0])
    with pytest.raises(TypeError):
        binding.cross_attn_fwd(q.half(), k, k, cq, ck, 4, 6, 0.1)


def data(seed, lq=(3, 0, 5), rows=(4, 2, 6), hq=4, hkv=2, d=8):
    rng = np.random.default_rng(seed)
    cq, ck = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(rows)])
    new = lambda t, h: rng.standard_normal((int(t), h, d))
    return new(cq[-1], hq), new(ck[-1], hkv), new(ck[-1], hkv), new(cq[-1], hq), cq, ck


def test_reference_against_self_attention():
    """The last query of a sequence sees all its keys: there both attentions are the same."""
    rng = np.random.default_rng(1)
    cu = np.array([0, 5, 12], dtype=np.int32)
    q, k, v = (rng.standard_normal((12, h, 64)).astype(np.float32) for h in (4, 2, 2))
    o, lse = attn_oracle.fwd(q, k, v, cu, 0.3)
    last = [4, 11]
    oc, lc = co.fwd(q[last], k, v, [0, 1, 2], cu, 0.3)
    np.testing.assert_allclose(oc, np.asarray(o)[last], atol=1e-12)
    np.testing.assert_allclose(lc, np.asarray(lse)[:, last], atol=1e-12)


def test_reference_closed_forms():
    q, k, v, do, cq, ck = data(2)
    o, lse = co.fwd(0 * q, k, v, cq, ck, 0.5)
    np.testing.assert_allclose(o[0, 0], v[:4, 0].mean(0), atol=1e-14)
    np.testing.assert_allclose(lse[:, 3:], np.log(6.0), atol=1e-14)
    o, lse = co.fwd(q, k, v, cq, ck, 0.5, kv_lens=[0, 1, 99])
    assert np.all(o[:3] == 0) and np.all(lse[:, :3] == -np.inf)
    o2, _ = co.fwd(q, k, v, cq, ck, 0.5)
    np.testing.assert_array_equal(o[3:], o2[3:])
    dq, dk, dv = co.bwd(q, k, v, o, lse, do, cq, ck, 0.5, kv_lens=[0, 1, 99])
    assert np.all(dq[:3] == 0) and np.all(dk[:6] == 0) and np.all(dv[:6] == 0)
    np.testing.assert_allclose(dv[6:].sum(0)[0], do[3:, :2].sum((0, 1)), atol=1e-12)      # rows of P sum to one
    np.testing.assert_allclose(dk[6:].sum(0), 0, atol=1e-12)                                # a shift of all keys changes nothing


def test_reference_against_differences():
    q, k, v, do, cq, ck = data(3)
    lens = [3, 2, 9]
    loss = lambda q, k, v: (co.fwd(q, k, v, cq, ck, 0.7, lens)[0] * do).sum()
    o, lse = co.fwd(q, k, v, cq, ck, 0.7, lens)
    grads = co.bwd(q, k, v, o, lse, do, cq, ck, 0.7, lens)
    rng = np.random.default_rng(4)
    for which, g in enumerate(grads):
        for _ in range(12):
            x = [a.copy() for a in (q, k, v)]
            at = tuple(int(rng.integers(0, n)) for n in g.shape)
            h = 1e-5
            x[which][at] += h
            up = loss(*x)
            x[which][at] -= 2 * h
            assert abs((up - loss(*x)) / (2 * h) - g[at]) < 1e-7
