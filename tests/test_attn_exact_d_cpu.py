"""The bounds of tests/_attn_exact_d.py against the arithmetic of the bf16 backward, done
by torch on the CPU: the corrected forms stay within them, forms that leave a correction
out do not."""
import pytest
import torch

from _attn_exact_d import CASES, SCALE, gradients, inputs
from _attn_ref import check


def bf(x):
    return x.bfloat16().float()


def arithmetic(q, k, v, do, scale, fix_dq, fix_dk):
    """dq and dk in fp32 with the roundings to bf16 that the kernels make."""
    B, Sq, H, D = q.shape
    G, rep = k.shape[2], q.shape[2] // k.shape[2]
    qh, doh = (x.float().permute(0, 2, 1, 3) for x in (q, do))
    kh, vh = (x.float().permute(0, 2, 1, 3).repeat_interleave(rep, 1) for x in (k, v))
    s = qh @ kh.transpose(-1, -2) * scale
    p = torch.exp(s - torch.logsumexp(s, -1, keepdim=True))
    out = bf(bf(p) @ vh)
    dp = doh @ vh.transpose(-1, -2)
    d = (doh * out).sum(-1, keepdim=True)
    ds = p * (dp - d)
    off = ds.sum(-1, keepdim=True)
    dq = bf(ds) @ kh
    if fix_dq:
        dq = dq - off * (bf(p) @ kh)
    ds = p * (dp - (d + off)) if fix_dk else ds
    dk = bf(ds).transpose(-1, -2) @ qh
    dk = dk.reshape(B, G, rep, -1, D).sum(2)
    return {"dq": (dq * scale).bfloat16().permute(0, 2, 1, 3),
            "dk": (dk * scale).bfloat16().permute(0, 2, 1, 3)}


@pytest.mark.parametrize("case", CASES, ids=str)
def test_bounds_hold_with_the_corrections_and_not_without(case):
    q, k, v, do = inputs(*case)
    want = gradients(q, k, v, do, scale=SCALE)
    got = arithmetic(q, k, v, do, SCALE, True, True)
    for n in want:
        check(n, got[n], want[n])
    got = arithmetic(q, k, v, do, SCALE, False, False)
    for n in want:
        with pytest.raises(AssertionError, match="beyond their bound"):
            check(n, got[n], want[n])
