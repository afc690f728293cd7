"""Rotary positions, self-attention and cross attention together, as a decoder layer of an encoder-decoder model runs them: forward,
backward, captured in a graph, on several streams, and one token at a time.

    q, k, v = parts of a fused projection;  q, k turned by their positions;  o1 = causal self-attention;  the queries o1 then look at
    the encoder's states ek, ev, rows of a padded buffer;  loss = <o2, w>

against torch's differentiation of the same formulas in fp64 on the CPU.

Tolerances are on norms.  fp32: an operator's relative error is at most 2 e + (n + d) 2^-24 of sums of absolute values, e = (d + 4)
2^-24 |score| <= 7e-5 for d = 64 and scores up to 16; those sums exceed the value's norm by sqrt(n) <= 18 at most, and five operators
follow each other: 5 * 18 * 1.7e-4 = 1.5e-2 bounds it.  bf16: an operator's output is off by 3.1e-3 of its norm (two roundings); a
query off by that moves scores of up to 4 sigma = 4 by 1.2e-2 and so every P, and the outputs behind it, by that of themselves;
the gradient of the first operators comes through three of those: 0.05 bounds it."""
import math

import numpy as np
import pytest
import torch

from paper_2412_07894_amd import binding

pytestmark = pytest.mark.gpu

LQ, ROWS, LENS = [5, 130, 1, 0, 300], [40, 333, 7, 64, 190], [33, 333, 0, 64, 150]
TOL = {torch.bfloat16: 0.05, torch.float32: 1.5e-2}


class Layer:
    def __init__(self, dtype, hq, hkv, d, rot, layout, seed=0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *shape: torch.randn(shape, generator=g).to(dtype).cuda()
        self.hq, self.hkv, self.d, self.rot, self.layout, self.dtype = hq, hkv, d, rot, layout, dtype
        self.cq = torch.tensor(np.concatenate([[0], np.cumsum(LQ)]), dtype=torch.int32, device="cuda")
        self.ck = torch.tensor(np.concatenate([[0], np.cumsum(ROWS)]), dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
        self.T, self.Tk, self.scale = sum(LQ), sum(ROWS), 1.0 / math.sqrt(d)
        self.qkv = rnd(self.T, hq + 2 * hkv, d)
        self.ek, self.ev, self.w = rnd(self.Tk, hkv, d), rnd(self.Tk, hkv, d), rnd(self.T, hq, d)
        self.freqs = binding.rope_frequencies(rot, scaling="parts", factor=4.0, original_length=64, low=1.0, high=4.0)
        self.dq_kv = torch.zeros_like(self.qkv)

    def forward(self, stream=None):
        s = dict(stream=stream)
        q, k, v = self.qkv.split([self.hq, self.hkv, self.hkv], dim=1)
        self.v = v.contiguous()
        self.q1, self.k1 = binding.rope_rotate(q, self.freqs, k=k, cu_seqlens=self.cq, layout=self.layout, magnitude=1.1, **s)
        self.o1, self.l1 = binding.varlen_attn_fwd(self.q1, self.k1, self.v, self.cq, max(LQ), self.scale, **s)
        self.o2, self.l2 = binding.cross_attn_fwd(self.o1, self.ek, self.ev, self.cq, self.ck, max(LQ), max(LENS), self.scale, kv_lens=self.lens, **s)
        return self.o2

    def backward(self, stream=None):
        s = dict(stream=stream)
        do1, dek, dev = binding.cross_attn_bwd(self.o1, self.ek, self.ev, self.o2, self.l2, self.w, self.cq, self.ck, max(LQ), max(LENS),
                                               self.scale, kv_lens=self.lens, **s)
        dq1, dk1, dv = binding.varlen_attn_bwd(self.q1, self.k1, self.v, self.o1, self.l1, do1, self.cq, max(LQ), self.scale, **s)
        a, b = self.hq, self.hq + self.hkv
        dqkv = self.dq_kv
        binding.rope_rotate(dq1, self.freqs, k=dk1, cu_seqlens=self.cq, layout=self.layout, magnitude=1.1, inverse=True,
                            out=dqkv[:, :a], k_out=dqkv[:, a:b], **s)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            dqkv[:, b:].copy_(dv)
        return dqkv, dek, dev

    def reference(self):
        """(o2, gradients of qkv, ek, ev) in fp64 on the CPU."""
        cpu = lambda t: t.detach().double().cpu()
        qkv, ek, ev = (cpu(t).requires_grad_() for t in (self.qkv, self.ek, self.ev))
        f, half, G = cpu(self.freqs), self.rot // 2, self.hq // self.hkv

        def turn(x, pos):
            ang = torch.as_tensor(pos, dtype=torch.float64)[:, None, None] * f
            c, s = ang.cos(), ang.sin()
            r, rest = x[..., :self.rot], x[..., self.rot:]
            if self.layout == "half":
                a, b = r[..., :half], r[..., half:]
                y = torch.cat([a * c - b * s, b * c + a * s], -1)
            else:
                a, b = r[..., 0::2], r[..., 1::2]
                y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
            return torch.cat([1.1 * y, rest], -1)

        def attn(q, k, v, causal):
            k, v = (t.repeat_interleave(G, 1).transpose(0, 1).contiguous() for t in (k, v))
            s = torch.matmul(q.transpose(0, 1), k.transpose(1, 2)) * self.scale
            if causal:
                s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool).triu(1), -math.inf)
            return torch.matmul(s.softmax(-1), v).transpose(0, 1)

        outs = []
        for i, (L, n) in enumerate(zip(LQ, LENS)):
            t0, k0 = int(self.cq[i]), int(self.ck[i])
            q, k, v = qkv[t0:t0 + L].split([self.hq, self.hkv, self.hkv], dim=1)
            pos = np.arange(L)
            o = attn(turn(q, pos), turn(k, pos), v, True)
            outs.append(attn(o, ek[k0:k0 + n], ev[k0:k0 + n], False) if n else 0.0 * o)
        o2 = torch.cat(outs)
        (o2 * cpu(self.w)).sum().backward()
        return o2.detach(), qkv.grad, ek.grad, ev.grad


def off(a, ref):
    return float((a.double().cpu() - ref).norm() / ref.norm())


SHAPES = [(torch.bfloat16, 8, 2, 128, 128, "half"), (torch.bfloat16, 4, 4, 64, 32, "interleaved"), (torch.float32, 6, 3, 64, 64, "half")]


@pytest.mark.parametrize("dtype,hq,hkv,d,rot,layout", SHAPES)
def test_forward_and_backward(dtype, hq, hkv, d, rot, layout):
    layer = Layer(dtype, hq, hkv, d, rot, layout)
    ref = layer.reference()
    got = (layer.forward(), *layer.backward())
    for name, a, b in zip(("o2", "d(qkv)", "d(ek)", "d(ev)"), got, ref):
        assert off(a, b) < TOL[dtype], (name, off(a, b))


def test_graph():
    """Forward and backward in one graph, replayed on other inputs, with eager calls between."""
    layer, eager = (Layer(torch.bfloat16, 8, 2, 128, 64, "half") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(), layer.backward()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = (layer.forward(), *layer.backward())
    for rep in range(4):
        for name in ("qkv", "ek", "ev", "w"):
            x = torch.randn(getattr(layer, name).shape, generator=torch.Generator().manual_seed(rep)).cuda()
            getattr(layer, name).copy_(x), getattr(eager, name).copy_(x)
        want = (eager.forward(), *eager.backward())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep


def test_two_streams_at_once():
    """Two layers on two streams give what each gives alone; nothing is shared between calls."""
    layers = [Layer(torch.bfloat16, 8, 2, 128, 64, "half", seed=1), Layer(torch.bfloat16, 4, 4, 64, 64, "half", seed=2)]
    want = [[x.clone() for x in (l.forward(), *l.backward())] for l in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(3):
        got = []
        for l, s in zip(layers, streams):
            l.v.zero_()
            l.dq_kv.zero_()
        torch.cuda.synchronize()
        for l, s in zip(layers, streams):
            with torch.cuda.stream(s):
                got.append((l.forward(stream=s), *l.backward(stream=s)))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_one_token_at_a_time():
    """The last token of every request by itself, at its position, gives what the whole pass gives for it: bit for bit in the rotation,
    within two roundings of O (2^-8 of P and of O each) in the attention."""
    layer = Layer(torch.bfloat16, 8, 2, 128, 128, "half")
    layer.forward()
    some = [i for i, L in enumerate(LQ) if L > 0]
    last = torch.tensor([int(layer.cq[i + 1]) - 1 for i in some], device="cuda")
    cu1 = torch.arange(len(some) + 1, dtype=torch.int32, device="cuda")
    starts = torch.tensor([LQ[i] - 1 for i in some], dtype=torch.int32, device="cuda")
    q, k, _ = layer.qkv.split([8, 2, 2], dim=1)
    q1, k1 = binding.rope_rotate(q[last].contiguous(), layer.freqs, k=k[last].contiguous(), cu_seqlens=cu1, starts=starts, magnitude=1.1)
    assert torch.equal(q1, layer.q1[last]) and torch.equal(k1, layer.k1[last])
    # the padded buffer as it lies: a request's rows by their first and last one, the rows of requests that are over by empty sequences
    cu_q = torch.tensor([sum(L > 0 for L in LQ[:i]) for i in range(len(LQ) + 1)], dtype=torch.int32, device="cuda")
    o, lse = binding.cross_attn_fwd(layer.o1[last].contiguous(), layer.ek, layer.ev, cu_q, layer.ck, 1, max(LENS), layer.scale, kv_lens=layer.lens)
    want = layer.o2[last].float()
    most = layer.ev.float().abs().max()
    assert torch.all((o.float() - want).abs() <= 2 * 2.0 ** -8 * (want.abs() + most))
    close = (lse - layer.l2[:, last]).abs() <= 1e-4
    assert torch.all(close | (lse == layer.l2[:, last]))
