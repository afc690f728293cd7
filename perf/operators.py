"""Cross attention of packed batches and rotary positions: the cases they are measured on, their
plain forms, and their definitions in 64 bits.

Every case is a dict of plain values; the lengths of its sequences follow from its `shape` number
alone, the values of its tensors from the seed.  `own` selects this repository's kernels."""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0


# ---- cases ------------------------------------------------------------------------------------

def _rope(name, seqs, lo, hi, starts, hq, hkv, d, rot, layout, scaling, dtype, inverse=False, fused=False, magnitude=1.0, shape=1):
    return {"name": name, "op": "rope", "seqs": seqs, "len_min": lo, "len_max": hi, "starts": starts, "hq": hq, "hkv": hkv, "d": d,
            "rot": rot, "layout": layout, "scaling": scaling, "dtype": dtype, "inverse": inverse, "fused": fused,
            "magnitude": magnitude, "shape": shape}


def _cross(name, op, seqs, q, kv, hq, hkv, d, dtype="bf16", empty=0, padded=False, shape=1):
    return {"name": name, "op": op, "seqs": seqs, "q_min": q[0], "q_max": q[1], "kv_min": kv[0], "kv_max": kv[1], "hq": hq, "hkv": hkv,
            "d": d, "dtype": dtype, "empty": empty, "padded": padded, "shape": shape}


def listed():
    return [
        # one new token of each running request, far into a context that was stretched four times: latency
        _rope("rope one token each", 16, 1, 1, 30000, 32, 8, 128, 128, "half", "parts", "bf16", magnitude=1.1),
        # a packed training batch straight out of the fused projection, Q and K together
        _rope("rope packed batch", 12, 64, 8192, 0, 32, 8, 128, 128, "half", "parts", "bf16", fused=True, shape=2),
        # the gradients of Q and K of a model that turns neighbouring pairs of the first half of each head
        _rope("rope gradients interleaved", 9, 100, 6000, 0, 40, 40, 128, 64, "interleaved", "plain", "bf16", inverse=True, shape=3),
        # a numerical check in fp32, a head and a turned part that are no power of two
        _rope("rope fp32 odd heads", 37, 1, 400, 0, 7, 1, 80, 24, "half", "linear", "fp32", shape=4),
        # transcription: one token each against a few seconds to half a minute of sound, the smallest attention call
        _cross("cross one token each", "cross_fwd", 4, (1, 1), (1500, 1500), 20, 20, 64),
        # serving: one token of each of 64 requests against long documents in a padded cache
        _cross("cross padded cache", "cross_fwd", 64, (1, 1), (500, 8192), 32, 8, 128, padded=True, shape=5),
        # a training batch of speech and transcripts, two clips without sound
        _cross("cross ragged batch", "cross_fwd", 24, (1, 448), (1, 1500), 20, 20, 64, empty=2, shape=6),
        # long documents and long answers
        _cross("cross long", "cross_fwd", 6, (1500, 6000), (4000, 12000), 32, 8, 128, shape=7),
        # gradients of the training batch
        _cross("cross gradients ragged", "cross_bwd", 24, (1, 448), (1, 1500), 20, 20, 64, empty=2, shape=6),
        # gradients of an image model that looks at a prompt: many rows, few keys
        _cross("cross gradients few keys", "cross_bwd", 16, (1024, 4096), (8, 77), 8, 8, 64, shape=8),
        # gradients of long documents and long answers
        _cross("cross gradients long", "cross_bwd", 4, (1500, 6000), (4000, 12000), 32, 8, 128, shape=9),
        # gradients of a numerical check in fp32
        _cross("cross gradients fp32", "cross_bwd", 7, (1, 500), (1, 900), 8, 2, 128, dtype="fp32", empty=1, shape=10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.randrange(1, 1 << 30)
    if rng.random() < 0.35:
        d = rng.choice([64, 128, 128, 80, 96, 256])
        rot = rng.choice([d, d, d // 2, 2 * rng.randrange(1, d // 2 + 1)])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 8])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        one = rng.random() < 0.3
        tokens = _log(rng, 1, 256) if one else _log(rng, 64, 40000)
        tokens = max(1, min(tokens, 200_000_000 // ((hq + hkv) * d)))
        seqs = tokens if one else min(_log(rng, 1, 64), tokens)
        mean = max(1, tokens // seqs)
        return {"op": "rope", "seqs": seqs, "len_min": 1 if one else max(1, mean // 4), "len_max": 1 if one else max(1, 7 * mean // 4),
                "starts": rng.choice([0, 1000, 100000]) if one else 0, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
                "layout": rng.choice(["half", "interleaved"]), "scaling": rng.choice(["plain", "linear", "parts"]), "dtype": dtype,
                "inverse": rng.random() < 0.4, "fused": rng.random() < 0.3, "magnitude": rng.choice([1.0, 1.0, 1.25]), "shape": shape}
    op = rng.choice(["cross_fwd", "cross_fwd", "cross_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    d = rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8, 10, 20])
    hq = hkv * rng.choice([1, 1, 2, 4] if hkv > 4 else [1, 2, 4, 8])
    seqs = _log(rng, 1, 64)
    one = op == "cross_fwd" and rng.random() < 0.4
    q_max = rng.choice([1, 1, rng.randrange(2, 20)]) if one else _log(rng, 8, 6000)
    kv_max = _log(rng, 8, 12000)
    q_min, kv_min = max(1, q_max // rng.randrange(1, 9)), max(1, kv_max // rng.randrange(1, 9))
    most = 1.2e8 if dtype == "bf16" else 2e6                         # (query, key) pairs of a head, times heads / 32 (fewer products in fp32)
    room = most * 32 / hq * (1 if op == "cross_fwd" else 0.5)
    while seqs > 1 and (seqs * q_max * kv_max > room or seqs * (q_max * hq + kv_max * hkv) * d > 3e8):
        seqs = (seqs + 1) // 2
    while q_max * kv_max > room:
        if q_max > kv_max:
            q_max = (q_max + 1) // 2
        else:
            kv_max = (kv_max + 1) // 2
    return {"op": op, "seqs": seqs, "q_min": min(q_min, q_max), "q_max": q_max, "kv_min": min(kv_min, kv_max), "kv_max": kv_max, "hq": hq,
            "hkv": hkv, "d": d, "dtype": dtype, "empty": 1 if seqs > 2 and rng.random() < 0.3 else 0, "padded": rng.random() < 0.3,
            "shape": shape}


# ---- lengths ----------------------------------------------------------------------------------

def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _rope_lens(case):
    rng = random.Random(case["shape"])
    lens = [_log(rng, case["len_min"], case["len_max"]) for _ in range(case["seqs"])]
    starts = [rng.randrange(case["starts"]) if case["starts"] else 0 for _ in lens]
    return lens, starts


def _cross_lens(case):
    """Query lengths, key lengths, and the rows that each sequence has in the key buffer."""
    rng = random.Random(case["shape"])
    n = case["seqs"]
    ql = [rng.randint(case["q_min"], case["q_max"]) for _ in range(n)]
    kl = [rng.randint(case["kv_min"], case["kv_max"]) for _ in range(n)]
    for s in rng.sample(range(n), case["empty"]):
        kl[s] = 0
    return ql, kl, [case["kv_max"]] * n if case["padded"] else kl


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        tokens, heads = sum(_rope_lens(case)[0]), case["hq"] + case["hkv"]
        return {"bytes": 2 * size * tokens * heads * case["d"], "flops": 3 * tokens * heads * case["rot"]}
    ql, kl, _ = _cross_lens(case)
    pairs = sum(a * b for a, b in zip(ql, kl)) * case["hq"]
    rows, keys = sum(ql) * case["hq"], sum(kl) * case["hkv"]
    if case["op"] == "cross_fwd":
        return {"bytes": size * case["d"] * (2 * rows + 2 * keys) + 4 * rows, "flops": 4 * case["d"] * pairs}
    return {"bytes": size * case["d"] * (4 * rows + 4 * keys) + 4 * rows, "flops": 10 * case["d"] * pairs}


# ---- inputs -----------------------------------------------------------------------------------

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _scaling(case):
    """Keywords of the frequencies: a context of 8192 positions, stretched four times."""
    if case["scaling"] == "linear":
        return {"scaling": "linear", "factor": 4.0}
    if case["scaling"] == "parts":
        return {"scaling": "parts", "factor": 4.0, "original_length": 8192.0, "low": 1.0, "high": 32.0}
    return {}


def _plain_frequencies(case):
    rot, sc = case["rot"], _scaling(case)
    out = []
    for i in range(rot // 2):
        f = BASE ** (-2.0 * i / rot)
        if case["scaling"] == "linear":
            f = f / sc["factor"]
        elif case["scaling"] == "parts":
            turns = sc["original_length"] * f / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - sc["low"]) / (sc["high"] - sc["low"])))
            f = f * keep + f / sc["factor"] * (1.0 - keep)
        out.append(f)
    return out


def _rope_inputs(case, seed):
    lens, starts = _rope_lens(case)
    cu = _cu(lens)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], TYPES[case["dtype"]]
    if case["fused"]:
        qkv = torch.randn((cu[-1], hq + 2 * hkv, d), generator=g, device=DEV, dtype=dt)
        q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    else:
        q = torch.randn((cu[-1], hq, d), generator=g, device=DEV, dtype=dt)
        k = torch.randn((cu[-1], hkv, d), generator=g, device=DEV, dtype=dt)
    return {"lens": lens, "starts": starts, "cu": cu, "q": q, "k": k}


def _cross_inputs(case, seed):
    ql, kl, rows = _cross_lens(case)
    cq, ck = _cu(ql), _cu(rows)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    d, dt = case["d"], TYPES[case["dtype"]]
    st = {"ql": ql, "kl": kl, "cq": cq, "ck": ck, "scale": 1.0 / math.sqrt(d)}
    st["q"] = torch.randn((cq[-1], case["hq"], d), generator=g, device=DEV, dtype=dt)
    st["k"] = torch.randn((ck[-1], case["hkv"], d), generator=g, device=DEV, dtype=dt)
    st["v"] = torch.randn((ck[-1], case["hkv"], d), generator=g, device=DEV, dtype=dt)
    if case["padded"]:                                               # what lies behind the valid keys of a cache is anything
        for s, n in enumerate(kl):
            st["k"][ck[s] + n:ck[s + 1]] = float("nan")
            st["v"][ck[s] + n:ck[s + 1]] = float("nan")
    if case["op"] == "cross_bwd":
        st["do"] = torch.randn(st["q"].shape, generator=g, device=DEV, dtype=dt)
        st["o"], st["lse"] = _plain_cross_fwd(st)                    # what the forward left
    return st


def prepare(case, seed):
    st = _rope_inputs(case, seed) if case["op"] == "rope" else _cross_inputs(case, seed)
    st["case"] = case
    if case["op"] == "rope":
        st["cu_dev"] = _ints(st["cu"])
        st["starts_dev"] = _ints(st["starts"]) if case["starts"] else None
        if own:
            from paper_2412_07894_amd import binding
            st["freqs"] = binding.rope_frequencies(case["rot"], BASE, device=DEV, **_scaling(case))
            st["q_out"] = torch.empty(st["q"].shape, dtype=st["q"].dtype, device=DEV)
            st["k_out"] = torch.empty(st["k"].shape, dtype=st["k"].dtype, device=DEV)
        else:
            pos = [a + i for a, n in zip(st["starts"], st["lens"]) for i in range(n)]
            st["pos"] = torch.tensor(pos, dtype=torch.float64, device=DEV)
            st["freqs"] = torch.tensor(_plain_frequencies(case), dtype=torch.float64, device=DEV)
        return st
    st["cq_dev"], st["ck_dev"] = _ints(st["cq"]), _ints(st["ck"])
    st["kl_dev"] = _ints(st["kl"]) if case["padded"] else None
    st["max_q"], st["max_kv"] = max(st["ql"]), max(max(b - a for a, b in zip(st["ck"], st["ck"][1:])), 1)
    if own:
        from paper_2412_07894_amd import binding
        bwd = case["op"] == "cross_bwd"
        need = binding.cross_attn_workspace_bytes(st["cq"][-1], st["ck"][-1], case["seqs"], st["max_q"], st["max_kv"], case["hq"],
                                                  case["hkv"], case["d"], binding.HYD_BF16 if case["dtype"] == "bf16" else binding.HYD_FP32, bwd)
        st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        if bwd:
            st["dq"], st["dk"], st["dv"] = torch.empty_like(st["q"]), torch.empty_like(st["k"]), torch.empty_like(st["v"])
        else:
            st["out"] = torch.empty_like(st["q"])
            st["lse_out"] = torch.empty((case["hq"], st["cq"][-1]), dtype=torch.float32, device=DEV)
    return st


# ---- plain forms ------------------------------------------------------------------------------

def _plain_rope(x, st, case):
    rot = case["rot"]
    ang = st["pos"][:, None] * st["freqs"][None, :]
    c = (torch.cos(ang) * case["magnitude"]).float()[:, None, :]
    s = (torch.sin(-ang if case["inverse"] else ang) * case["magnitude"]).float()[:, None, :]
    y = x.float()
    if case["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(x.dtype)


MOST = 1 << 28                                                       # scores that are held at once


def _pieces(st, s, heads_kv, group):
    """(first KV head, last one, first row, last row) of pieces of sequence s with at most MOST scores."""
    n, rows = max(st["kl"][s], 1), max(st["ql"][s], 1)
    heads = max(1, min(heads_kv, MOST // (rows * group * n)))
    step = max(1, min(rows, MOST // (heads * group * n)))
    for g in range(0, heads_kv, heads):
        for r in range(0, st["ql"][s], step):
            yield g, min(heads_kv, g + heads), r, min(st["ql"][s], r + step)


def _rows(x, a, b, g0, g1, group):
    """Rows a..b of the query heads of KV heads g0..g1: [KV heads, (row, head of the group), d] in 32 bits."""
    y = x[a:b, g0 * group:g1 * group].float()
    return y.reshape(b - a, g1 - g0, group, -1).transpose(0, 1).reshape(g1 - g0, (b - a) * group, -1)


def _back(y, rows, group):
    """Inverse of _rows: [row, query heads, d]."""
    g = y.shape[0]
    return y.reshape(g, rows, group, -1).transpose(0, 1).reshape(rows, g * group, -1)


def _plain_cross_fwd(st):
    q, k, v = st["q"], st["k"], st["v"]
    hkv, group = k.shape[1], q.shape[1] // k.shape[1]
    o = torch.zeros_like(q)
    lse = torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float32, device=DEV)
    for s, n in enumerate(st["kl"]):
        if n == 0:
            continue
        ka, qa = st["ck"][s], st["cq"][s]
        for g0, g1, r0, r1 in _pieces(st, s, hkv, group):
            ks = k[ka:ka + n, g0:g1].float().transpose(0, 1).contiguous()
            vs = v[ka:ka + n, g0:g1].float().transpose(0, 1).contiguous()
            x = torch.matmul(_rows(q, qa + r0, qa + r1, g0, g1, group), ks.transpose(1, 2)) * st["scale"]
            top = x.amax(dim=-1, keepdim=True)
            x = torch.exp(x - top)
            total = x.sum(dim=-1, keepdim=True)
            y = torch.matmul(x, vs) / total
            o[qa + r0:qa + r1, g0 * group:g1 * group] = _back(y, r1 - r0, group).to(o.dtype)
            lse[g0 * group:g1 * group, qa + r0:qa + r1] = _back(top + torch.log(total), r1 - r0, group)[..., 0].t()
    return o, lse


def _plain_cross_bwd(st):
    q, k, v, o, do = st["q"], st["k"], st["v"], st["o"], st["do"]
    hkv, group = k.shape[1], q.shape[1] // k.shape[1]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for s, n in enumerate(st["kl"]):
        if n == 0:
            continue
        ka, qa = st["ck"][s], st["cq"][s]
        sums = {}
        for g0, g1, r0, r1 in _pieces(st, s, hkv, group):
            ks = k[ka:ka + n, g0:g1].float().transpose(0, 1).contiguous()
            vs = v[ka:ka + n, g0:g1].float().transpose(0, 1).contiguous()
            qs, dos, os = (_rows(x, qa + r0, qa + r1, g0, g1, group) for x in (q, do, o))
            ls = st["lse"][g0 * group:g1 * group, qa + r0:qa + r1].reshape(g1 - g0, group, r1 - r0).transpose(1, 2).reshape(g1 - g0, -1, 1)
            p = torch.exp(torch.matmul(qs, ks.transpose(1, 2)) * st["scale"] - ls)
            ds = p * (torch.matmul(dos, vs.transpose(1, 2)) - (dos * os).sum(dim=-1, keepdim=True))
            dq[qa + r0:qa + r1, g0 * group:g1 * group] = _back(torch.matmul(ds, ks) * st["scale"], r1 - r0, group).to(dq.dtype)
            part = torch.matmul(ds.transpose(1, 2), qs) * st["scale"], torch.matmul(p.transpose(1, 2), dos)
            sums[g0, g1] = tuple(a + b for a, b in zip(sums[g0, g1], part)) if (g0, g1) in sums else part
        for (g0, g1), (a, b) in sums.items():
            dk[ka:ka + n, g0:g1] = a.transpose(0, 1).to(dk.dtype)
            dv[ka:ka + n, g0:g1] = b.transpose(0, 1).to(dv.dtype)
    return dq, dk, dv


def run(st):
    case = st["case"]
    if case["op"] == "rope":
        if own:
            from paper_2412_07894_amd import binding
            q, k = binding.rope_rotate(st["q"], st["freqs"], k=st["k"], cu_seqlens=st["cu_dev"], starts=st["starts_dev"],
                                       layout=case["layout"], magnitude=case["magnitude"], inverse=case["inverse"],
                                       out=st["q_out"], k_out=st["k_out"])
        else:
            q, k = _plain_rope(st["q"], st, case), _plain_rope(st["k"], st, case)
        return {"q": q, "k": k}
    if case["op"] == "cross_fwd":
        if own:
            from paper_2412_07894_amd import binding
            o, lse = binding.cross_attn_fwd(st["q"], st["k"], st["v"], st["cq_dev"], st["ck_dev"], st["max_q"], st["max_kv"],
                                            st["scale"], kv_lens=st["kl_dev"], workspace=st["ws"], out=st["out"], lse=st["lse_out"])
        else:
            o, lse = _plain_cross_fwd(st)
        return {"o": o, "lse": lse}
    if own:
        from paper_2412_07894_amd import binding
        dq, dk, dv = binding.cross_attn_bwd(st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], st["cq_dev"], st["ck_dev"],
                                            st["max_q"], st["max_kv"], st["scale"], kv_lens=st["kl_dev"], workspace=st["ws"],
                                            dq=st["dq"], dk=st["dk"], dv=st["dv"])
    else:
        dq, dk, dv = _plain_cross_bwd(st)
    return {"dq": dq, "dk": dk, "dv": dv}


# ---- definitions in 64 bits ---------------------------------------------------------------------

def _exact_rope(case, seed):
    st = _rope_inputs(case, seed)
    rot, half = case["rot"], case["rot"] // 2
    if case["layout"] == "half":
        first, second = torch.arange(half, device=DEV), torch.arange(half, device=DEV) + half
    else:
        first, second = 2 * torch.arange(half, device=DEV), 2 * torch.arange(half, device=DEV) + 1
    f = torch.pow(torch.tensor(BASE, dtype=torch.float64, device=DEV), -torch.arange(half, dtype=torch.float64, device=DEV) * 2 / rot)
    sc = _scaling(case)
    if case["scaling"] == "linear":
        f = f / sc["factor"]
    elif case["scaling"] == "parts":
        keep = ((sc["original_length"] * f / (2 * math.pi) - sc["low"]) / (sc["high"] - sc["low"])).clamp(0, 1)
        f = keep * f + (1 - keep) * f / sc["factor"]
    pos = torch.cat([torch.arange(a, a + n, dtype=torch.float64) for a, n in zip(st["starts"], st["lens"])]).to(DEV)
    turn = torch.polar(torch.full((pos.numel(), half), case["magnitude"], dtype=torch.float64, device=DEV), torch.outer(pos, f))
    if case["inverse"]:
        turn = turn.conj()
    out = {}
    for name in ("q", "k"):
        y = st[name].double()
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None, :]
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def _exact_cross(case, seed):
    st = _cross_inputs(case, seed)
    q, k, v, hq, group = st["q"], st["k"], st["v"], case["hq"], case["hq"] // case["hkv"]
    bwd = case["op"] == "cross_bwd"
    wide = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    if bwd:
        dq, dk, dv = wide(q), wide(k), wide(v)
    else:
        o, lse = wide(q), torch.full((hq, q.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    for s, n in enumerate(st["kl"]):
        if n == 0:
            continue
        keys = slice(st["ck"][s], st["ck"][s] + n)
        for h in range(hq):
            kh, vh = k[keys, h // group].double(), v[keys, h // group].double()
            for a in range(st["cq"][s], st["cq"][s + 1], max(1, (1 << 27) // n)):
                rows = slice(a, min(st["cq"][s + 1], a + max(1, (1 << 27) // n)))
                x = (q[rows, h].double() @ kh.t()) * st["scale"]
                if not bwd:
                    ls = torch.logsumexp(x, dim=1)
                    o[rows, h], lse[h, rows] = torch.exp(x - ls[:, None]) @ vh, ls
                    continue
                doh = st["do"][rows, h].double()
                p = torch.exp(x - st["lse"][h, rows].double()[:, None])
                ds = p * (doh @ vh.t() - (doh * st["o"][rows, h].double()).sum(1, keepdim=True))
                dq[rows, h] = st["scale"] * (ds @ kh)
                dk[keys, h // group] += st["scale"] * (ds.t() @ q[rows, h].double())
                dv[keys, h // group] += p.t() @ doh
    return {"dq": dq, "dk": dk, "dv": dv} if bwd else {"o": o, "lse": lse}


def exact(case, seed):
    return _exact_rope(case, seed) if case["op"] == "rope" else _exact_cross(case, seed)
