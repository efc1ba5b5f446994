"""The attention operators where values or shapes are at an edge: biases beyond fp32's
exponent, queries behind the last one and queries that see no key."""
import pytest
import torch

import paper_2202_11836_amd as P
from _attn_ref import check, reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(shape, seed, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).cuda()


def both(q, k, v, do, relpos=None, **kw):
    """Forward and backward: results by name."""
    rp = P.RelPos(*relpos) if relpos else None
    out, lse = P.attn_forward(q, k, v, relpos=rp, **kw)
    got = dict(zip(("dq", "dk", "dv", "dtable"),
                   P.attn_backward(q, k, v, out, lse, do, relpos=rp, **kw)), out=out, lse=lse)
    torch.cuda.synchronize()
    return got


# (batch, heads, key heads, queries, keys): one launch for the whole backward; two, by the
# number of work-groups and by the number of keys; two wavefronts to 32 queries and one
SHAPES = [(2, 2, 2, 33, 70), (2, 4, 2, 70, 33), (17, 16, 16, 33, 40), (2, 2, 1, 70, 450),
          (9, 16, 16, 300, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("relpos,causal", [((32, 128, True), False), ((8, 20, True), False),
                                           ((32, 128, False), True)])
def test_biases_beyond_the_exponent(dtype, shape, relpos, causal):
    """A constant added to the bias is none to the softmax, however large: exp(100) is
    beyond fp32, and a work-group has lanes behind the last query whose log-sum-exp nothing
    takes off."""
    B, H, G, Sq, Sk = shape
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    table = rand((relpos[0], H), 5) + 100.0
    kw = dict(table=table, causal=causal)
    got = both(q, k, v, do, relpos=relpos, **kw)
    want = reference(q, k, v, relpos=relpos, dout=do, **kw)
    for n in want:
        check(n, got[n], want[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES + [(2, 6, 2, 150, 190), (1, 4, 4, 600, 700)], ids=str)
@pytest.mark.parametrize("relpos", [None, (32, 128, False), (8, 20, True)])
@pytest.mark.parametrize("left", [False, True])
def test_queries_that_see_no_key(dtype, shape, relpos, left):
    """Before position 0, and before the first key that a mask leaves (sequences padded
    at their left), a query's q and dout may hold anything."""
    B, H, G, Sq, Sk = shape
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    pos = torch.tensor([(-21, 5, -1, 0, -64)[b % 5] for b in range(B)], dtype=torch.int32)
    first = torch.zeros(B, dtype=torch.int32)  # visible key
    mask = None
    if left:
        first = torch.tensor([(0, 17, 32, Sk - 1, Sk)[b % 5] for b in range(B)], dtype=torch.int32)
        mask = (torch.arange(Sk)[None, :] >= first[:, None]).to(torch.uint8).cuda()
    none = (torch.arange(Sq)[None, :] + pos[:, None] < first[:, None]).cuda()
    none |= (first == Sk)[:, None].cuda()
    assert none.any() and not none.all()
    table = rand((relpos[0], H), 5) if relpos else None
    kw = dict(causal=True, q_pos=pos.cuda(), key_mask=mask, table=table)
    bad_q, bad_do = q.clone(), do.clone()
    bad_q[none], bad_do[none] = float("inf"), float("nan")
    got = both(bad_q, k, v, bad_do, relpos=relpos, **kw)
    q[none], do[none] = 0, 0
    kw["mask"] = kw.pop("key_mask")
    want = reference(q, k, v, relpos=relpos, dout=do, **kw)
    for n in want:
        check(n, got[n], want[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tables_gradient_left_out(dtype):
    """dtable=False with a table, without one (where there is none to make), and into given
    tensors."""
    q, do = rand((2, 33, 4, 64), 1, dtype), rand((2, 33, 4, 64), 2, dtype)
    k, v = rand((2, 50, 2, 64), 3, dtype), rand((2, 50, 2, 64), 4, dtype)
    rp, table = P.RelPos(8, 20), rand((8, 4), 5)
    for kw in (dict(relpos=rp, table=table), {}):
        out, lse = P.attn_forward(q, k, v, **kw)
        to = [torch.full_like(t, float("nan")) for t in (q, k, v)]
        got = P.attn_backward(q, k, v, out, lse, do, dq=to[0], dk=to[1], dv=to[2], dtable=False, **kw)
        assert got[3] is None and all(a is b for a, b in zip(got, to))
        want = reference(q, k, v, dout=do, relpos=(8, 20, True) if kw else None,
                         table=kw.get("table"))
        for n, g in zip(("dq", "dk", "dv"), got):
            check(n, g, want[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES + [(2, 4, 2, 1, 300)], ids=str)
@pytest.mark.parametrize("low", [float("-inf"), torch.finfo(torch.float32).min])
def test_biases_that_hide(dtype, shape, low):
    """Buckets of -inf, or of fp32's lowest value, hide their keys in both passes, far and
    near: here those behind the query, and, where a query has no others, all of them."""
    B, H, G, Sq, Sk = shape
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    pos = torch.tensor([(0, -20, 7)[b % 3] for b in range(B)], dtype=torch.int32)
    table = rand((8, H), 5)
    hidden = table.clone()
    hidden[4:] = low  # (8 buckets both ways: from 4 on of keys behind the query)
    got = both(q, k, v, do, relpos=(8, 20, True), table=hidden, q_pos=pos.cuda())
    want = reference(q, k, v, relpos=(8, 20, True), dout=do, table=table, q_pos=pos.cuda(), causal=True)
    for n in want:
        check(n, got[n], want[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 1), (10, 2)])
@pytest.mark.parametrize("relpos", [None, (32, 128, False)])
def test_long_paddings_at_the_left(dtype, heads, kv, relpos):
    """Sequences of up to 600 tokens padded at their left by whole blocks and more, whose
    padding holds anything in every operand."""
    first = [300, 130, 512, 0, 599]
    B, S = len(first), 600
    pad = (torch.arange(S)[None, :] < torch.tensor(first)[:, None]).cuda()
    q, do = rand((B, S, heads, 64), 1, dtype), rand((B, S, heads, 64), 2, dtype)
    k, v = rand((B, S, kv, 64), 3, dtype), rand((B, S, kv, 64), 4, dtype)
    table = rand((relpos[0], heads), 5) if relpos else None
    bad = [t.clone() for t in (q, k, v, do)]
    for t, x in zip(bad, ("nan", "inf", "nan", "-inf")):
        t[pad] = float(x)
    mask = (~pad).to(torch.uint8)
    got = both(*bad, relpos=relpos, key_mask=mask, causal=True, table=table)
    for t in (q, k, v, do):
        t[pad] = 0
    want = reference(q, k, v, mask=mask, relpos=relpos, dout=do, causal=True, table=table)
    for n in want:
        check(n, got[n], want[n])
