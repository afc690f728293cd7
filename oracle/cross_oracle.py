"""TEST INFRASTRUCTURE ONLY - plain fp64 reference of cross attention over packed batches, forward and backward.

    sequence s: queries are rows [cu_q[s], cu_q[s+1]), keys rows [cu_kv[s], cu_kv[s] + n_s), n_s = min(kv_lens[s], cu_kv[s+1] - cu_kv[s])
    s_ij = scale <Q_i, K_j>;  LSE_i = ln sum_j exp(s_ij);  O_i = sum_j exp(s_ij - LSE_i) V_j;  n_s = 0: O = 0, LSE = -inf
    backward of given (O, LSE):  P = exp(s - LSE), D_i = <dO_i, O_i>, dS = P (<dO_i, V_j> - D_i)
       dQ = scale dS K;  dK = scale sum over the group's heads of dS^T Q;  dV = sum of P^T dO;  keys behind the valid ones: 0

Dense numpy per (sequence, head).  Rows of no sequence are nan.  Only tests/ may import this module.
"""
import numpy as np


def _seqs(cu_q, cu_kv, kv_lens):
    for s in range(len(cu_q) - 1):
        a, b, c, e = int(cu_q[s]), int(cu_q[s + 1]), int(cu_kv[s]), int(cu_kv[s + 1])
        n = e - c if kv_lens is None else max(0, min(int(kv_lens[s]), e - c))
        yield a, b, c, e, n


def fwd(q, k, v, cu_q, cu_kv, scale, kv_lens=None):
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    Tq, hq, d = q.shape
    group = hq // k.shape[1]
    o, lse = np.full((Tq, hq, d), np.nan), np.full((hq, Tq), np.nan)
    for a, b, c, e, n in _seqs(cu_q, cu_kv, kv_lens):
        for h in range(hq):
            if n == 0:
                o[a:b, h], lse[h, a:b] = 0.0, -np.inf
                continue
            x = scale * (q[a:b, h] @ k[c:c + n, h // group].T)
            m = x.max(axis=1, keepdims=True) if b > a else np.zeros((0, 1))
            p = np.exp(x - m)
            total = p.sum(axis=1, keepdims=True)
            o[a:b, h] = (p / total) @ v[c:c + n, h // group]
            lse[h, a:b] = (m + np.log(total))[:, 0]
    return o, lse


def bwd(q, k, v, o, lse, do, cu_q, cu_kv, scale, kv_lens=None):
    q, k, v, o, lse, do = (np.asarray(x, dtype=np.float64) for x in (q, k, v, o, lse, do))
    hq, group = q.shape[1], q.shape[1] // k.shape[1]
    dq, dk, dv = np.full(q.shape, np.nan), np.full(k.shape, np.nan), np.full(v.shape, np.nan)
    for a, b, c, e, n in _seqs(cu_q, cu_kv, kv_lens):
        dq[a:b], dk[c:e], dv[c:e] = 0.0, 0.0, 0.0
        if n == 0 or a == b:
            continue
        for h in range(hq):
            g = h // group
            p = np.exp(scale * (q[a:b, h] @ k[c:c + n, g].T) - lse[h, a:b, None])
            ds = p * (do[a:b, h] @ v[c:c + n, g].T - (do[a:b, h] * o[a:b, h]).sum(axis=1, keepdims=True))
            dq[a:b, h] = scale * (ds @ k[c:c + n, g])
            dk[c:c + n, g] += scale * (ds.T @ q[a:b, h])
            dv[c:c + n, g] += p.T @ do[a:b, h]
    return dq, dk, dv
