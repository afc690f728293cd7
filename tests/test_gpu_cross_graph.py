"""Cross attention captured once and replayed on other lengths: a graph holds the sizes and bounds of its call, everything else follows
from the device arrays at the time of the replay."""
import numpy as np
import pytest
import torch

from paper_2412_07894_amd import binding
from cross_util import DT, cu_of

pytestmark = pytest.mark.gpu


def split(rng, total, n, most, front):
    """n lengths up to `most` with a sum of at most total - front."""
    left, out = total - front, []
    for _ in range(n):
        out.append(int(rng.integers(0, min(most, left) + 1)))
        left -= out[-1]
    return cu_of(out, front)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,max_q,max_kv,hq,hkv", [(6, 2, 3000, 8, 2), (5, 60, 100, 4, 4), (5, 60, 2500, 2, 2), (40, 130, 900, 6, 3), (90, 300, 260, 8, 8)])
def test_lengths_change_between_replays(n, max_q, max_kv, hq, hkv, dtype):
    d, scale = 64, 0.125
    Tq, Tk = n * max_q // 2 + 7, n * max_kv // 2 + 5
    rng = np.random.default_rng(n)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    new = lambda t, h: torch.randn((t, h, d), generator=g, device="cuda").to(DT[dtype])
    q, k, v, do = new(Tq, hq), new(Tk, hkv), new(Tk, hkv), new(Tq, hq)
    cq, ck = (torch.from_numpy(split(rng, t, n, m, 0)).cuda() for t, m in ((Tq, max_q), (Tk, max_kv)))
    lens = torch.full((n,), max_kv, dtype=torch.int32, device="cuda")
    code = binding.HYD_BF16 if dtype == "bf16" else binding.HYD_FP32
    need = [binding.cross_attn_workspace_bytes(Tq, Tk, n, max_q, max_kv, hq, hkv, d, code, b) for b in (False, True)]

    class Call:
        def __init__(self):
            self.ws = [torch.empty(x, dtype=torch.uint8, device="cuda") for x in need]
            self.out = [torch.empty_like(q), torch.empty((hq, Tq), device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]

        def run(self):
            a = (cq, ck, max_q, max_kv, scale)
            o, lse, dq, dk, dv = self.out
            binding.cross_attn_fwd(q, k, v, *a, kv_lens=lens, workspace=self.ws[0], out=o, lse=lse)
            binding.cross_attn_bwd(q, k, v, o, lse, do, *a, kv_lens=lens, workspace=self.ws[1], dq=dq, dk=dk, dv=dv)

    eager, held = Call(), Call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.run()
    for rep in range(5):
        front = int(rng.integers(0, 4))
        cq.copy_(torch.from_numpy(split(rng, Tq, n, max_q, front)))
        ck.copy_(torch.from_numpy(split(rng, Tk, n, max_kv, front)))
        lens.copy_(torch.from_numpy(rng.integers(-1, max_kv + 2, n).astype(np.int32)))
        for c in (eager, held):
            for x in c.out:
                x.fill_(7.0)
        for w in held.ws:
            w.fill_(255 if rep % 2 else 0)
        eager.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), held.out, eager.out):
            assert torch.equal(a, b), (rep, name)
