"""Bounds for the bf16 gradients dq and dk that hold only where the rounding of a bf16
`out` does not reach D (tests/_attn_ref.py allows it).

With p, dp, D, g = p (dp - D) exact, u = 2^-24, t = 2^-8 (half a step of bf16), ep the
relative error of P and e_dp that of a product dout . v:
  - D formed from P and dP, or D' = rowsum(dout * out) + off with off = sum_j P (dp - D'):
    both are sum_j P dp up to (1 - sum_j P) D', so
        e_D = sum_j p (ep (|dp| + |D|) + e_dp + (Sk + 4) u (|dp| + |D|))
  - dk takes P (dp - D) rounded to bf16: off by p e_D and t of the value;
  - dq, with D' = D + delta, |delta| <= sum |dout| (the error of out): sum_j of
    bf16(P (dp - D')) k - off bf16(P) k.  delta cancels but for the two roundings:
    t p |delta| for each of them.
"""
import torch

U, T = 2.0 ** -24, 2.0 ** -8


def gradients(q, k, v, do, mask=None, scale=0.125, causal=False, bias=None):
    """q, do [B, Sq, H, 64], k, v [B, Sk, G, 64] bf16, bias [H, Sq, Sk] or None ->
    {"dq", "dk": (value, bound)} in float64 on the CPU."""
    q, k, v, do = (x.detach().cpu().double() for x in (q, k, v, do))
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1], k.shape[2]
    rep = H // G
    qh, doh = q.permute(0, 2, 1, 3), do.permute(0, 2, 1, 3)
    kh, vh = (x.permute(0, 2, 1, 3).repeat_interleave(rep, 1) for x in (k, v))
    vis = torch.ones(B, 1, Sq, Sk, dtype=torch.bool)
    if mask is not None:
        vis &= (mask.cpu() != 0)[:, None, None, :]
    if causal:
        vis &= torch.ones(Sq, Sk, dtype=torch.bool).tril()
    vis = vis.expand(B, H, Sq, Sk)
    s = qh @ kh.transpose(-1, -2) * scale
    ds = U * 68 * scale * (qh.abs() @ kh.abs().transpose(-1, -2))
    if bias is not None:
        bias = bias.detach().cpu().double()
        s, ds = s + bias, ds + 3 * U * bias.abs()
    s = torch.where(vis, s, torch.full((), -torch.inf).double())
    lse = torch.logsumexp(s, -1, keepdim=True)  # (every row of these tests sees a key)
    p = torch.exp(s - lse)
    ds = torch.where(vis, ds + 4 * U * s.abs().nan_to_num(posinf=0.0), 0.0)
    ep = ds + ds.amax(-1, keepdim=True) + U * (8 + Sk + 4 * lse.abs())
    out = p @ vh
    e_out = (p * (ep + T + Sk * U)) @ vh.abs()
    e_out = e_out * (1 + T) + T * out.abs()
    delta = (doh.abs() * (e_out + 66 * U * out.abs())).sum(-1, keepdim=True)
    dp = doh @ vh.transpose(-1, -2)
    Dm = (p * dp).sum(-1, keepdim=True)
    size = dp.abs() + Dm.abs()
    e_dp = 66 * U * (doh.abs() @ vh.abs().transpose(-1, -2) + Dm.abs())
    e_D = (p * (ep * size + e_dp + (Sk + 4) * U * size)).sum(-1, keepdim=True)
    g = p * (dp - Dm)
    e_g = p * (e_dp + e_D + 2 * U * size) + (ep + 2 * U) * g.abs()
    e_g = e_g + T * (g.abs() + e_g)
    e_q = e_g + 2 * T * p * (delta + e_D) + Sk * U * (g.abs() + 2 * p * delta)
    dq = g @ kh * scale
    e = e_q @ kh.abs() * scale
    e = e * (1 + T + 2 * U) + T * dq.abs()

    def fold(x):
        return x.reshape(B, G, rep, Sk, D).sum(2).permute(0, 2, 1, 3)

    dk = fold(g.transpose(-1, -2) @ qh * scale)
    ek = fold((e_g + rep * Sq * U * g.abs()).transpose(-1, -2) @ qh.abs() * scale)
    return {"dq": (dq.permute(0, 2, 1, 3), e.permute(0, 2, 1, 3)),
            "dk": (dk, ek * (1 + T + 2 * U) + T * dk.abs())}


# (batch, heads, key heads, queries, keys): one launch (the first two); two; two with the
# keys of dQ split over work-groups (of 1000 and 3000 keys)
CASES = [(2, 4, 2, 9, 17), (3, 4, 4, 77, 201), (2, 2, 2, 40, 500), (9, 16, 16, 200, 130),
         (2, 4, 1, 300, 260), (2, 2, 2, 40, 1000), (1, 2, 1, 25, 3000)]


def inputs(B, H, G, Sq, Sk):
    """bf16, on the CPU; scores of some units, so that a few keys take most of P and dS is
    of the size of what out's rounding adds to it."""
    g = torch.Generator().manual_seed(Sq + Sk)

    def n(*shape):
        return torch.randn(*shape, generator=g).bfloat16()

    return n(B, Sq, H, 64), n(B, Sk, G, 64), n(B, Sk, G, 64), n(B, Sq, H, 64)


SCALE = 0.75
