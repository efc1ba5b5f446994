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
