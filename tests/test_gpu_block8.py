"""A block of a model in 8 bits, every operator as it is used with the others: norm -> gated product pair -> activation -> product -> norm with gate into
the residual stream, and back.

The reference is the block in float64 on the CPU, with codes formed by the same rule and gradients that pass a code's rounding by, the activation's slope taken
at the checkpoint.  Tolerance: a number that float32 has off by 40 u takes the next code where its quotient is that close to a border, which 2 * 127 * 40 u =
6e-4 of all numbers are; each then is off by 1 / 127 of its row's largest, some 3 % of the row's root mean square, so a tensor of codes by
sqrt(6e-4) * 0.03 = 7e-4 of itself.  Five such tensors in a row, and the sums of products behind them, each passing it on with a factor near 1: 5e-3 is held.
"""
import math

import pytest
import torch

from paper_2501_02379_amd import act8, norms

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


class Block:
    """x' = x + alpha g (norm(down(silu(gate(h)) up(h))) w_post),  h = norm(x) w_pre;  then h' = norm(x') w_next."""

    def __init__(self, width, hidden, seed=0, dtype=torch.float32):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.wide = r(2 * hidden, width) / math.sqrt(width)              # both products of the gated pair in one
        self.down = r(width, hidden) / math.sqrt(hidden)
        self.pre, self.post, self.next = (1 + 0.1 * r(width) for _ in range(3))
        self.gate = 0.7 + 0.2 * r(1, width)
        self.alpha, self.hidden, self.dtype = 0.5, hidden, dtype

    def to_gpu(self):
        self.wide8, self.down8 = (act8.tgrad_quantize(w.to(DEV)) for w in (self.wide, self.down))
        self.p, self.q, self.n = (w.to(DEV) for w in (self.pre, self.post, self.next))
        self.g = self.gate.to(self.dtype).to(DEV)
        return self

    def forward(self, x, **kw):
        f = self.hidden
        self.x, self.rows = x, x.shape[0]
        self.a = norms.tgrad_block_norm(x, pre_weight=self.p, eps=EPS, quantize=True, dtype=self.dtype, **kw)
        both = act8.tgrad_codes_matmul(self.a.h, self.wide8, dtype=self.dtype, **kw)
        self.act = act8.tgrad_activation(both[:, :f], both[:, f:], act="silu", group=64, quantize=True, **kw)
        self.out = act8.tgrad_codes_matmul(self.act.y, self.down8, dtype=self.dtype, **kw)
        self.b = norms.tgrad_block_norm(x, self.out, post_weight=self.q, gate=self.g, rows_per_gate=self.rows, scale=self.alpha, pre_weight=self.n, eps=EPS, **kw)
        return self.b.x, self.b.h

    def backward(self, dx, dh, **kw):
        r = norms.tgrad_block_norm_backward(dx, dh, self.b.x, self.out, stats=self.b.stats, post_weight=self.q, gate=self.g, rows_per_gate=self.rows,
                                            scale=self.alpha, pre_weight=self.n, **kw)
        dy = act8.tgrad_codes_grad_input(r.dblock, self.down8, **kw)
        ddown = act8.tgrad_codes_grad_weight(r.dblock, self.act.y, **kw)
        both = torch.empty(self.rows, 2 * self.hidden, dtype=self.dtype, device=DEV)
        act8.tgrad_activation_backward(dy, self.act.x8, self.act.gate8, out=both[:, :self.hidden], gate_out=both[:, self.hidden:], **kw)
        dh0 = act8.tgrad_codes_grad_input(both, self.wide8, **kw)
        dwide = act8.tgrad_codes_grad_weight(both, self.a.h, **kw)
        s = norms.tgrad_block_norm_backward(r.dx, dh0, self.x, stats=self.a.stats, pre_weight=self.p, **kw)
        return s.dx, dwide, ddown, r.dgate, s.dpre, r.dpost, r.dpre


def coded(v, group=0):
    """v as its codes say, in float64."""
    out = torch.empty_like(v)
    step = group or v.shape[1]
    for i in range(0, v.shape[1], step):
        p = v[:, i:i + step]
        top = p.abs().amax(1, keepdim=True)
        out[:, i:i + step] = torch.round(127 * p / top) * (top.float() / 127).double()
    return out


class Passing(torch.autograd.Function):
    """Codes whose rounding the gradient passes by."""
    @staticmethod
    def forward(ctx, v):
        return coded(v)

    @staticmethod
    def backward(ctx, d):
        return d


class Gated(torch.autograd.Function):
    """silu(a) b with the gradient of what the checkpoint says a and b are."""
    @staticmethod
    def forward(ctx, a, b):
        ctx.save_for_backward(coded(a, 64), coded(b, 64))
        return torch.nn.functional.silu(a) * b

    @staticmethod
    def backward(ctx, d):
        a, b = ctx.saved_tensors
        p = torch.sigmoid(a)
        return d * b * p * (1 + a * (1 - p)), d * a * p


def reference(m, x, dx, dh):
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    x, wide, down, pre, post, nxt, gate = map(leaf, (x, m.wide, m.down, m.pre, m.post, m.next, m.gate))
    norm = lambda v: v * (v.square().mean(1, keepdim=True) + EPS).rsqrt()  # noqa: E731
    both = Passing.apply(norm(x) * pre) @ Passing.apply(wide).t()
    y = Passing.apply(Gated.apply(both[:, :m.hidden], both[:, m.hidden:])) @ Passing.apply(down).t()
    out = x + m.alpha * gate * (norm(y) * post)
    h = norm(out) * nxt
    ((out * dx.double()).sum() + (h * dh.double()).sum()).backward()
    return (out, h), (x.grad, wide.grad, down.grad, gate.grad, pre.grad, post.grad, nxt.grad)


@pytest.mark.parametrize("rows,width,hidden", [(1, 64, 96), (37, 130, 200), (300, 256, 320), (513, 129, 257)])
def test_a_block_forward_and_backward(rows, width, hidden):
    m = Block(width, hidden).to_gpu()
    g = torch.Generator().manual_seed(9)
    x, dx, dh = (torch.randn(rows, width, generator=g) for _ in range(3))
    got = m.forward(x.to(DEV))
    grads = m.backward(dx.to(DEV), dh.to(DEV))
    want, want_grads = reference(m, x, dx, dh)
    for a, b in zip(got + grads, want + want_grads):
        b = b.detach()
        assert a.shape == b.shape
        assert float((a.cpu().double() - b).norm() / b.norm()) <= 5e-3


def test_a_block_in_bf16_captured_and_on_another_stream():
    rows = 400
    m = Block(256, 512, dtype=torch.bfloat16).to_gpu()
    g = torch.Generator().manual_seed(9)
    x, dx, dh = (torch.randn(rows, 256, generator=g).bfloat16().to(DEV) for _ in range(3))
    run = lambda **kw: m.forward(x, **kw) + m.backward(dx, dh, **kw)  # noqa: E731
    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    held = []
    for graph in graphs:                                                # two of them, replayed in turn
        with torch.cuda.graph(graph):
            held.append(run())
    for i in range(4):
        x.mul_(1.25)
        graphs[i % 2].replay()
        want = run()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        for got in held:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
