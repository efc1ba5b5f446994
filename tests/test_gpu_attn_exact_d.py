"""bf16 gradients dq and dk within bounds that the rounding of `out` in D would break
(tests/test_attn_exact_d_cpu.py shows that it would)."""
import pytest
import torch

import paper_2202_11836_amd as P
from _attn_exact_d import CASES, SCALE, gradients, inputs
from _attn_ref import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_rounding_of_out_stays_out_of_d(case, mask, causal):
    q, k, v, do = (x.cuda() for x in inputs(*case))
    m = None
    if mask:  # (key 0 stays, for the first query of `causal`)
        m = (torch.rand((case[0], case[4]), generator=torch.Generator().manual_seed(1)) < 0.7)
        m[:, 0] = True
        m = m.to(torch.uint8).cuda()
    kw = dict(key_mask=m, scale=SCALE, causal=causal)
    out, lse = P.attn_forward(q, k, v, **kw)
    dq, dk, _, _ = P.attn_backward(q, k, v, out, lse, do, **kw)
    torch.cuda.synchronize()
    want = gradients(q, k, v, do, mask=m, scale=SCALE, causal=causal)
    print({n: round(check(n, g, want[n]), 3) for n, g in (("dq", dq), ("dk", dk))}, flush=True)


# (one launch for the backward; two, by the number of work-groups and of keys; chunks of
# queries, whose sums follow)
@pytest.mark.parametrize("case", [(2, 4, 4, 128, 128), (9, 16, 16, 200, 130), (2, 4, 2, 150, 700),
                                  (2, 8, 2, 70, 130)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_without_the_tables_gradient(case, causal):
    """dtable=False: the other gradients are those of a call that makes it, within bounds
    that out's rounding would break, and None stands for it."""
    B, H, G, Sq, Sk = case
    q, k, v, do = (x.cuda() for x in inputs(*case))
    rp = P.RelPos(32, 128)
    table = torch.randn(32, H, generator=torch.Generator().manual_seed(3)).cuda()
    kw = dict(scale=SCALE, causal=causal, relpos=rp, table=table)
    out, lse = P.attn_forward(q, k, v, **kw)
    dq, dk, dv, dt = P.attn_backward(q, k, v, out, lse, do, dtable=False, **kw)
    full = P.attn_backward(q, k, v, out, lse, do, **kw)
    torch.cuda.synchronize()
    assert dt is None and full[3] is not None
    ids = torch.tensor([[rp.bucket(j - i) for j in range(Sk)] for i in range(Sq)])
    bias = table.cpu()[ids].permute(2, 0, 1)
    want = gradients(q, k, v, do, scale=SCALE, causal=causal, bias=bias)
    for n, a, b in (("dq", dq, full[0]), ("dk", dk, full[1])):
        check(n, a, want[n])
        check(n, b, want[n])
    assert torch.equal(dv, full[2])
