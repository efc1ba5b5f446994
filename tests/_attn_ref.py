"""The attention operators in float64, straight from their formulas, with bounds
of the rounding errors that an implementation of the given type may make.

Units: u = 2^-24 (fp32, half a step relative to the value), t the half step of the
operands' type (bf16 2^-8, fp32 2^-24), which results are rounded to, and on bf16
the half step by which P and dS are rounded for the matrix products.
"""
import math

import torch

U = torch.finfo(torch.float32).eps / 2


def bucket(rel, num_buckets, max_distance, both):
    """Bucket of one distance, in whole numbers."""
    n = num_buckets // 2 if both else num_buckets
    base, d = (n, rel) if both and rel > 0 else (0, max(-rel, 0))
    one = n // 2
    m = n - one
    if d < one:
        return base + d
    d = min(d, max_distance)
    j = 0
    while j + 1 < m and d ** m * one ** (j + 1) >= one ** m * max_distance ** (j + 1):
        j += 1
    return base + one + j


def reference(q, k, v, mask=None, scale=0.125, causal=False, q_pos=None, relpos=None, table=None,
              dout=None):
    """q [B, Sq, H, D], k, v [B, Sk, G, D] (any type) -> {name: (value, bound)} in
    float64 on the CPU; relpos = (num_buckets, max_distance, both)."""
    t = torch.finfo(q.dtype).eps / 2
    p_round = t if q.dtype == torch.bfloat16 else 0.0
    out_type = q.dtype
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1], k.shape[2]
    rep = H // G
    qh = q.permute(0, 2, 1, 3)
    vis = torch.ones(B, Sq, Sk, dtype=torch.bool)
    if mask is not None:
        vis &= (mask.cpu() != 0)[:, None, :]
    pos = torch.zeros(B, dtype=torch.int64) if q_pos is None else q_pos.cpu().long()
    rel = torch.arange(Sk)[None, None, :] - (torch.arange(Sq)[None, :, None] + pos[:, None, None])
    if causal:
        vis &= rel <= 0
    # rows that no query sees may hold anything
    seen = vis.any(1)
    k = torch.where(seen[:, :, None, None], k, torch.zeros(()).double())
    v = torch.where(seen[:, :, None, None], v, torch.zeros(()).double())
    kh = k.permute(0, 2, 1, 3).repeat_interleave(rep, 1)
    vh = v.permute(0, 2, 1, 3).repeat_interleave(rep, 1)
    vis = vis[:, None].expand(B, H, Sq, Sk)
    s = qh @ kh.transpose(-1, -2) * scale
    # a sum of 64 products, the factor, the bias, the change to base 2
    ds = U * (68 * scale * (qh.abs() @ kh.abs().transpose(-1, -2)))
    ids = None
    if relpos is not None:
        lo, hi = int(rel.min()) if rel.numel() else 0, int(rel.max()) if rel.numel() else 0
        far = relpos[1]
        ids_of = {d: bucket(d, *relpos) for d in range(max(lo, -far), min(hi, far) + 1)}
        if lo < -far:
            ids_of[-far] = bucket(-far, *relpos)
        if hi > far:
            ids_of[far] = bucket(far, *relpos)
        first = min(ids_of) if ids_of else 0
        lut = torch.tensor([ids_of[d] for d in sorted(ids_of)] or [0])
        ids = lut[(rel.clamp(-far, far) - first)] if rel.numel() else rel
        bias = table.detach().cpu().double()[ids].permute(0, 3, 1, 2)
        s = s + bias
        ds = ds + 3 * U * bias.abs()
    s = torch.where(vis, s, torch.full((), -math.inf).double())
    lse = torch.logsumexp(s, -1) if Sk else torch.full((B, H, Sq), -math.inf).double()
    some = torch.isfinite(lse)[..., None]
    p = torch.where(vis & some, torch.exp(s - torch.where(some, lse[..., None], 0.0)), 0.0)
    # relative error of P: the scores' twice (score and log-sum-exp), the roundings
    # of the exponent's terms, the exponential and the sum (n terms)
    ds = torch.where(vis, ds + 4 * U * s.abs().nan_to_num(posinf=0.0), 0.0)
    worst = ds.amax(-1, keepdim=True) if Sk else torch.zeros(B, H, Sq, 1).double()
    lse_f = torch.where(some[..., 0], lse, 0.0)
    ep = ds + worst + U * (8 + Sk + 4 * lse_f.abs()[..., None])
    got = {"lse": (lse, worst[..., 0] + U * (8 + Sk + 2 * lse_f.abs()))}
    out = p @ vh
    e_out = (p * (ep + p_round + Sk * U)) @ vh.abs()
    e_out = e_out * (1 + t) + t * out.abs()
    got["out"] = (out.permute(0, 2, 1, 3), e_out.permute(0, 2, 1, 3))
    if dout is None:
        return got
    do = dout.detach().cpu().double().permute(0, 2, 1, 3)
    dp = do @ vh.transpose(-1, -2)
    e_dp = 66 * U * (do.abs() @ vh.abs().transpose(-1, -2))
    Dm = (p * dp).sum(-1, keepdim=True)
    # D from the rounded out, or (bf16 with a bias gradient) from P and dP
    e_D_out = (do.abs() * e_out).sum(-1, keepdim=True) + \
        66 * U * (do.abs() * out.abs()).sum(-1, keepdim=True)
    e_D_sum = (p * (ep * dp.abs() + e_dp + (Sk + 2) * U * dp.abs())).sum(-1, keepdim=True)
    exact_D = relpos is not None
    e_D = e_D_sum if exact_D and out_type == torch.bfloat16 else e_D_out
    g = p * (dp - Dm)
    e_g = p * (e_dp + e_D + 2 * U * (dp.abs() + Dm.abs())) + (ep + 2 * U) * g.abs()
    e_gr = e_g + p_round * (g.abs() + e_g)

    def fold(x):  # heads that share keys
        return x.reshape(B, G, rep, Sk, D).sum(2).permute(0, 2, 1, 3)

    def bound(val, err, n):
        return err * (1 + t) + n * U * err + t * val.abs()

    dq = (g @ kh) * scale
    e = (e_gr + Sk * U * g.abs()) @ kh.abs() * scale
    got["dq"] = (dq.permute(0, 2, 1, 3), bound(dq, e, 2).permute(0, 2, 1, 3))
    dk = fold(g.transpose(-1, -2) @ qh * scale)
    e = fold((e_gr + rep * Sq * U * g.abs()).transpose(-1, -2) @ qh.abs() * scale)
    got["dk"] = (dk, bound(dk, e, 2))
    dv = fold(p.transpose(-1, -2) @ do)
    e = fold((p * (ep + p_round + rep * Sq * U)).transpose(-1, -2) @ do.abs())
    got["dv"] = (dv, bound(dv, e, 2))
    if relpos is not None:
        nb = relpos[0]
        dt, de = torch.zeros(nb, H).double(), torch.zeros(nb, H).double()
        for h in range(H):
            dt[:, h] = torch.bincount(ids.reshape(-1), g[:, h].reshape(-1), minlength=nb)[:nb]
            # 64 + Sk + B additions at most lie between a term and its bucket's sum
            de[:, h] = torch.bincount(
                ids.reshape(-1), (e_g[:, h] + (64 + Sk + B) * U * g[:, h].abs()).reshape(-1),
                minlength=nb)[:nb]
        got["dtable"] = (dt, de)
    return got


def check(name, got, want, extra=0.0):
    """Every element of got within the bound of (value, bound); infinities equal."""
    val, err = want
    x = got.detach().cpu().double()
    assert x.shape == val.shape, (name, x.shape, val.shape)
    inf = torch.isinf(val)
    assert torch.equal(x[inf], val[inf]), f"{name}: infinities differ"
    off = (x - val).abs()[~inf]
    lim = err[~inf] * (1 + 1e-6) + extra + 1e-30
    bad = ~(off <= lim)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} beyond their bound, worst "
                           f"{float((off / lim).nan_to_num(nan=math.inf).max()):.3g} times; nan "
                           f"{int(torch.isnan(x).sum())}")
    return float((off / lim).max()) if off.numel() else 0.0
