"""A training step as a program makes it of the operators: layer norm, projections, rotary
positions, attention, the way back, and AdamW; against the same step in float64."""
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import rand

pytestmark = pytest.mark.gpu


def model64(x, w, ga, be, pos0):
    """x [B, S, 128] -> x + attention(rotary(LN(x) W)), 2 heads, in float64 with autograd."""
    B, S, C = x.shape
    d = x - x.mean(-1, keepdim=True)
    y = ga * d * ((d * d).mean(-1, keepdim=True) + 1e-5).rsqrt() + be
    q, k, v = (y @ w.t()).view(B, S, 3, 2, 64).unbind(2)
    f = 10000.0 ** (-torch.arange(16, dtype=torch.float64, device=x.device) / 16)
    a = (torch.arange(S, device=x.device).double()[None, :] + pos0.double()[:, None])[:, :, None, None] * f

    def turn(t):
        t0, t1 = t[..., :16], t[..., 16:32]
        return torch.cat([t0 * a.cos() - t1 * a.sin(), t0 * a.sin() + t1 * a.cos(), t[..., 32:]], -1)

    sc = (turn(q).transpose(1, 2) @ turn(k).transpose(1, 2).transpose(-1, -2).contiguous()) / 8
    o = (torch.softmax(sc, -1) @ v.transpose(1, 2)).transpose(1, 2).reshape(B, S, C)
    return x + o


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps(bits):
    """Three steps in fp32.  A gradient is off by a few hundred roundings of its terms; AdamW's
    update of a weight is at most 3 lr a step, and off by its gradient's relative error or, where
    the gradient is below the error, by all of it: so the weights' moves agree to 1e-3 in the
    2-norm (8 bits: the first step, whose states were 0)."""
    B, S, C = 3, 37, 128
    x, dy, ga, be = rand((B, S, C), 1), rand((B, S, C), 2), 1 + rand((C,), 3, std=0.1), rand((C,), 4, std=0.1)
    w = rand((3 * C, C), 5, std=0.05)
    pos0 = torch.tensor([0, 5, 900], dtype=torch.int32, device="cuda")
    rot = P.Rotary(32)
    params = [w, ga, be]
    ref = [t.double().requires_grad_() for t in params]
    ref_opt = torch.optim.AdamW(ref, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.05)
    grads = [torch.zeros_like(t) for t in params]
    opt = P.AdamW(params, grads, weight_decay=0.05, state_bits=bits)
    start = [t.clone() for t in params]
    for step in range(3 if bits == 32 else 1):
        y, total, mean, rstd = P.layer_norm_forward(x, ga, be, eps=1e-5)
        qkv = (y.view(-1, C) @ w.t()).view(B, S, 3, 2, 64)
        q, k, v = qkv.unbind(2)
        P.rotary_forward(rot, q, k, pos=pos0, q_out=q, k_out=k)
        o, lse = P.attn_forward(q, k, v)
        out = x + o.reshape(B, S, C)
        want = model64(x.double(), *ref, pos0)
        assert (out - want).abs().max() < 1e-4
        d = torch.empty_like(qkv)
        dq, dk, dv = d.unbind(2)
        P.attn_backward(q, k, v, o, lse, dy.view(B, S, 2, 64), dq=dq, dk=dk, dv=dv)
        P.rotary_backward(rot, dq, dk, pos=pos0, q_out=dq, k_out=dk)
        d = d.view(-1, 3 * C)
        torch.mm(d.t(), y.view(-1, C), out=grads[0])
        dx, _, _ = P.layer_norm_backward((d @ w).view(B, S, C), total, ga, mean, rstd, dtotal=dy,
                                         dgamma=grads[1], dbeta=grads[2])
        xr = x.double().requires_grad_()
        got = torch.autograd.grad((model64(xr, *ref, pos0) * dy.double()).sum(), [xr] + ref)
        for name, a, b in zip(("dx", "dw", "dgamma", "dbeta"), [dx] + grads, got):
            assert ((a - b).norm() / b.norm()).item() < 1e-4, (step, name)
        for r, gr in zip(ref, got[1:]):
            r.grad = gr
        ref_opt.step()
        opt.step(1e-3)
        for s0, a, b in zip(start, params, ref):
            moved = (b.detach() - s0.double())
            assert ((a.double() - b.detach()).norm() / moved.norm()).item() < 1e-3 * (step + 1)


def test_captured_step():
    """The whole step in one graph, its own workspaces and states; replays follow their inputs and
    equal eager steps bit for bit."""
    B, S, C = 2, 70, 128
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    rot = P.Rotary()

    class Run:
        def __init__(self):
            self.x = rand((B, S, C), 1, "bf16")
            self.w, self.ga = rand((3 * C, C), 5, "bf16", 0.05), torch.ones(C, device="cuda")
            self.be = torch.zeros(C, device="cuda")
            self.grads = [torch.zeros((3 * C, C), dtype=torch.bfloat16, device="cuda"),
                          torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")]
            self.opt = P.AdamW([self.w, self.ga, self.be], self.grads, state_bits=[8, 32, 32])

        def step(self):
            y, total, mean, rstd = P.layer_norm_forward(self.x, self.ga, self.be)
            qkv = (y.view(-1, C) @ self.w.t()).view(B, S, 3, 2, 64)
            q, k, v = qkv.unbind(2)
            q2, k2 = P.rotary_forward(rot, q, k, pos=pos)
            o, lse = P.attn_forward(q2, k2, v, causal=True)
            d = torch.empty_like(qkv)
            dq, dk, dv = d.unbind(2)
            P.attn_backward(q2, k2, v, o, lse, o, causal=True, dq=dq, dk=dk, dv=dv)
            P.rotary_backward(rot, dq, dk, pos=pos, q_out=dq, k_out=dk)
            d = d.view(-1, 3 * C)
            torch.mm(d.t(), y.view(-1, C), out=self.grads[0])
            P.layer_norm_backward((d @ self.w).view(B, S, C), total, self.ga, mean, rstd, dx=False,
                                  dgamma=self.grads[1], dbeta=self.grads[2])
            self.norm = self.opt.step(1e-3, max_norm=0.1)

    a, b = Run(), Run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.step()
    b.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        a.step()
    for i in range(1, 4):
        a.x.copy_(rand((B, S, C), 30 + i))
        b.x.copy_(a.x)
        pos.fill_(10 * i)
        g.replay()
        torch.cuda.synchronize()
        b.step()
        torch.cuda.synchronize()
        assert torch.equal(a.w, b.w) and torch.equal(a.ga, b.ga) and torch.equal(a.be, b.be), i
        assert torch.equal(a.norm, b.norm)
