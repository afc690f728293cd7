"""Shared by the tests of cross attention: inputs, calls through the binding, and tolerances from arithmetic.

bf16 forward.  A rounding to bf16 is off by at most u = 2^-8 of the value.  P is rounded once for the second product, O once: |dO| <=
u sum_j P_ij |V_j| + u |O|, and what the scores' fp32 sums (d terms, each 2^-24 of sum |q k|) and the exponentials add.
LSE: no rounding to bf16 enters; the scores' error and a few units of 2^-24 of its own size.

bf16 backward, given O and LSE.  P and dS are rounded to fp16 (h = 2^-11 of the value, 2^-25 absolutely below its normal range; dO is
scaled to a largest value in [1, 2), so there 2^-25 counts in units of that), results to bf16; in dK, dS is formed from a P that is
rounded already.  The scores' error e moves every P by e of itself, the fp32 sums of dP every dS by P times theirs; fp16 copies of
elements below 2^-14 keep 2^-25.
fp32: products and sums in fp32, d + n terms."""
import numpy as np
import torch

from oracle import cross_oracle as co
from paper_2412_07894_amd import binding

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def cu_of(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Case:
    """Packed inputs: lq queries and rows key rows of each sequence, valid keys kv_lens (None: all); front / back rows of no
    sequence; what lies behind the valid keys is nan, in padded rows and outside the sequences."""

    def __init__(self, lq, rows, hq, hkv, d, dtype="bf16", kv_lens=None, scale=None, seed=0, front=0, back=0, size=1.0):
        self.lq, self.rows, self.hq, self.hkv, self.d, self.dtype = list(lq), list(rows), hq, hkv, d, dtype
        self.kv_lens = None if kv_lens is None else list(kv_lens)
        self.scale = 1.0 / float(np.sqrt(d)) if scale is None else scale
        self.cq, self.ck = cu_of(lq, front), cu_of(rows, front)
        self.Tq, self.Tk = int(self.cq[-1]) + back, int(self.ck[-1]) + back
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        new = lambda T, h, s=1.0: (torch.randn((T, h, d), generator=g, device="cuda") * s).to(DT[dtype])
        self.q, self.k, self.v, self.do = new(self.Tq, hq, size), new(self.Tk, hkv, size), new(self.Tk, hkv), new(self.Tq, hq)
        self.n = [r if self.kv_lens is None else max(0, min(x, r)) for r, x in zip(self.rows, self.kv_lens or self.rows)]
        on = torch.zeros(self.Tk, dtype=torch.bool)
        for a, n in zip(self.ck[:-1], self.n):
            on[int(a):int(a) + n] = True
        for t in (self.k, self.v):
            t[~on.cuda()] = float("nan")
        self.q_rows = np.zeros(self.Tq, dtype=bool)
        self.q_rows[int(self.cq[0]):int(self.cq[-1])] = True
        self.kv_rows = np.zeros(self.Tk, dtype=bool)
        self.kv_rows[int(self.ck[0]):int(self.ck[-1])] = True
        for t in (self.q, self.do):
            t[~torch.from_numpy(self.q_rows).cuda()] = float("nan")
        self.cq_dev, self.ck_dev = torch.from_numpy(self.cq).cuda(), torch.from_numpy(self.ck).cuda()
        self.kl_dev = None if self.kv_lens is None else torch.tensor(self.kv_lens, dtype=torch.int32, device="cuda")
        self.max_q, self.max_kv = max(self.lq + [1]), max(self.n + [0])

    def args(self):
        return self.cq_dev, self.ck_dev, self.max_q, self.max_kv, self.scale

    def fwd(self, **kw):
        return binding.cross_attn_fwd(self.q, self.k, self.v, *self.args(), kv_lens=self.kl_dev, **kw)

    def bwd(self, o, lse, **kw):
        return binding.cross_attn_bwd(self.q, self.k, self.v, o, lse, self.do, *self.args(), kv_lens=self.kl_dev, **kw)

    def cpu(self):
        clean = lambda t: np.nan_to_num(np64(t), nan=0.0)
        return clean(self.q), clean(self.k), clean(self.v)


def _wide(c, x):
    return np.abs(x).max() if x.size else 0.0


def score_error(c):
    """Largest error of a score in fp32: d products and as many sums of at most |q| |k|, the scale, its product with log2(e)."""
    q, k, _ = c.cpu()
    big = abs(c.scale) * np.sqrt((q ** 2).sum(-1)).max(initial=0.0) * np.sqrt((k ** 2).sum(-1)).max(initial=0.0)
    return (c.d + 4) * 2.0 ** -24 * big


def check_fwd(c, o, lse, what=""):
    q, k, v = c.cpu()
    ref_o, ref_l = co.fwd(q, k, v, c.cq, c.ck, c.scale, c.kv_lens)
    abs_o, _ = co.fwd(q, k, np.abs(v), c.cq, c.ck, c.scale, c.kv_lens)
    o, lse = np64(o)[c.q_rows], np64(lse)[:, c.q_rows]
    ref_o, ref_l, abs_o = ref_o[c.q_rows], ref_l[:, c.q_rows], abs_o[c.q_rows]
    e, u = score_error(c), U[c.dtype]
    extra = 2.0 ** -20 if c.dtype == "bf16" else (max(c.n + [0]) + 8) * 2.0 ** -24        # exponentials and fp32 sums
    tol_o = (u + 2 * e + extra) * abs_o + u * (1 + u) * np.abs(ref_o) + 1e-30
    with np.errstate(invalid="ignore"):
        tol_l = e + 8 * 2.0 ** -24 * (np.abs(ref_l) + 1) + extra
        err_o, err_l = np.abs(o - ref_o), np.where(ref_l == lse, 0.0, np.abs(lse - ref_l))
    assert np.all(np.isfinite(o)), f"{what}: O is not finite"
    assert np.all(err_o <= tol_o), f"{what}: O off by {np.max(err_o / tol_o):.2f} of the bound"
    assert np.all(np.where(np.isinf(ref_l), lse == ref_l, err_l <= tol_l)), f"{what}: LSE off by {np.nanmax(err_l):.3e}"
    norm = np.sqrt((ref_o ** 2).sum())
    if c.dtype == "bf16" and norm > 0 and ref_o.size > 4096:
        # two roundings of 2^-8 / sqrt(3) * 0.74 each (errors uniform in a step, mantissas log-uniform), and a quarter more
        assert np.sqrt((err_o ** 2).sum()) / norm < 1.25 * np.sqrt(2) * 0.74 * 2.0 ** -8 / np.sqrt(3), what


def check_bwd(c, o, lse, dq, dk, dv, what=""):
    """Gradients against the reference's backward of the same O and LSE."""
    q, k, v = c.cpu()
    do, o, lse = (np.nan_to_num(np64(x), nan=0.0) for x in (c.do, o, lse))
    ref = co.bwd(q, k, v, o, lse, do, c.cq, c.ck, c.scale, c.kv_lens)
    tol = [np.zeros(x.shape) for x in (q, k, v)]
    bf = c.dtype == "bf16"
    u, h, tiny, e, group = U[c.dtype], 2.0 ** -11 if bf else 0.0, 2.0 ** -25 if bf else 0.0, score_error(c), c.hq // c.hkv
    big = np.abs(do[c.q_rows]).max(initial=0.0)
    for s, n in enumerate(c.n):
        rows, keys = slice(int(c.cq[s]), int(c.cq[s + 1])), slice(int(c.ck[s]), int(c.ck[s]) + n)
        if n == 0 or c.lq[s] == 0:
            continue
        acc = (max(n, c.lq[s] * group) + c.d) * 2.0 ** -24
        for hd in range(c.hq):
            g = hd // group
            Q, K, V, dO, O = q[rows, hd], k[keys, g], v[keys, g], do[rows, hd], o[rows, hd]
            L = lse[hd, rows, None]
            P = np.exp(c.scale * (Q @ K.T) - L)
            dP, D = dO @ V.T, (dO * O).sum(1, keepdims=True)
            dS = np.abs(P * (dP - D))
            e2 = 2 * e + 2.0 ** -21 * (1 + np.abs(L)) + acc
            # dP: its sums, fp16 copies of V and of the scaled dO that are below the normal range, D's sum
            edp = 2 * c.d * 2.0 ** -24 * (np.abs(dO) @ np.abs(V).T + np.abs(dO * O).sum(1, keepdims=True)) + tiny * (np.abs(dO).sum(1, keepdims=True) + big * np.abs(V).sum(1)[None])
            tol[0][rows, hd] += abs(c.scale) * (((h + e2) * dS + P * edp + 2 * tiny * big) @ (np.abs(K) + tiny))
            tol[1][keys, g] += abs(c.scale) * (((2 * h + e2) * dS + P * edp + tiny * np.abs(dP - D) + 4 * tiny * big).T @ (np.abs(Q) + tiny))
            tol[2][keys, g] += ((h + e2) * P + tiny).T @ np.abs(dO) + P.sum(0)[:, None] * tiny * big
    for name, got, r, t, on in zip(("dq", "dk", "dv"), (dq, dk, dv), ref, tol, (c.q_rows, c.kv_rows, c.kv_rows)):
        got, r, t = np64(got)[on], r[on], t[on]
        t = t + u * (1 + u) * np.abs(r) + 1e-30
        assert np.all(np.isfinite(got)), f"{what} {name} is not finite"
        err = np.abs(got - r)
        assert np.all(err <= t), f"{what} {name}: off by {np.max(err / t):.2f} of the bound"
        norm = np.sqrt((r ** 2).sum())
        if bf and norm > 0 and r.size > 4096:
            # one rounding of 2^-8 / sqrt(3) * 0.74, those to fp16 are an eighth of it; a quarter more
            rel = np.sqrt((err ** 2).sum()) / norm
            assert rel < 1.25 * 0.74 * 2.0 ** -8 / np.sqrt(3), f"{what} {name}: rel {rel:.3e}"
