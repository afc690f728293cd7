"""Self-attention backward with more heads than a block of its statistics holds (4096), against fp64 on the GPU."""
import pytest
import torch

from paper_2412_07894_amd import binding

pytestmark = pytest.mark.gpu


def dense(q, k, v, o, lse, do, cu, scale):
    """Gradients in fp64, a (sequence, KV head) at a time."""
    T, hq, d = q.shape
    hkv, G = k.shape[1], hq // k.shape[1]
    q, do, o = (x.double().view(T, hkv, G, d) for x in (q, do, o))
    k, v, lse = k.double(), v.double(), lse.double().t().reshape(T, hkv, G)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, b in zip(cu, cu[1:]):
        pos = torch.arange(b - a, device=q.device)
        seen = (pos[None, :] <= pos[:, None]).repeat_interleave(G, 0)
        for g in range(hkv):
            Q, D, O, L = q[a:b, g].reshape(-1, d), do[a:b, g].reshape(-1, d), o[a:b, g].reshape(-1, d), lse[a:b, g].reshape(-1, 1)
            p = torch.exp(scale * (Q @ k[a:b, g].t()) - L) * seen
            ds = p * (D @ v[a:b, g].t() - (D * O).sum(1, keepdim=True))
            dq[a:b, g] = (scale * (ds @ k[a:b, g])).view(-1, G, d)
            dk[a:b, g], dv[a:b, g] = scale * (ds.t() @ Q), p.t() @ D
    return dq.reshape(T, hq, d), dk, dv


@pytest.mark.parametrize("hq,hkv,d", [(9000, 3, 64), (20480, 1, 64), (4100, 2, 128), (4200, 4200, 64)])
@pytest.mark.parametrize("ranged", [False, True])
def test_backward(hq, hkv, d, ranged):
    cu, scale = [0, 3, 8, 9], 0.125
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rnd = lambda h: torch.randn((9, h, d), generator=g, device="cuda").to(torch.bfloat16)
    q, k, v, do = rnd(hq), rnd(hkv), rnd(hkv), rnd(hq)
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    o, lse = binding.varlen_attn_fwd(q, k, v, cud, 5, scale)
    if ranged:
        whole = torch.tensor([[0, 256, 0, 256]] * 3, dtype=torch.int32, device="cuda")
        got = [torch.empty_like(x) for x in (q, k, v)]
        binding.varlen_attn_bwd_range(q, k, v, o, lse, do, cud, whole, 5, scale, *got)
    else:
        got = binding.varlen_attn_bwd(q, k, v, o, lse, do, cud, 5, scale)
    for name, a, b in zip(("dq", "dk", "dv"), got, dense(q, k, v, o, lse, do, cu, scale)):
        # one rounding of 2^-8 / sqrt(3) * 0.74, those to fp16 are an eighth of it; a quarter more
        assert float((a.double() - b).norm() / b.norm()) < 1.25 * 0.74 * 2.0 ** -8 / 3 ** 0.5, name
