"""The attention operators on the GPU against float64, elementwise within the
rounding bounds of tests/_attn_ref.py: lengths from none to several blocks, masks,
layouts, shared key heads, relative position bias, single tokens."""
import pytest
import torch

import paper_2202_11836_amd as P
from _attn_ref import check, reference

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(dtype, B, H, G, Sq, Sk, seed=0, layout="plain"):
    """q, k, v, dout on the GPU.  layout: plain [B, S, H, D]; packed: k and v (and q
    for equal lengths and heads) side by side in one tensor; heads_first: [B, H, S, D]
    in memory; shared: one sequence of keys for the whole batch (stride 0)."""
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]

    def n(*shape):
        return torch.randn(*shape, generator=g).to(dt).cuda()

    if layout == "packed" and Sq == Sk and G == H:
        q, k, v = n(B, Sq, 3, H, 64).unbind(2)
    elif layout == "packed":
        q, (k, v) = n(B, Sq, H, 64), n(B, Sk, 2, G, 64).unbind(2)
    elif layout == "heads_first":
        q = n(B, H, Sq, 64).transpose(1, 2)
        k, v = n(B, G, Sk, 64).transpose(1, 2), n(B, G, Sk, 64).transpose(1, 2)
    elif layout == "shared":
        q = n(B, Sq, H, 64)
        k, v = n(1, Sk, G, 64).expand(B, -1, -1, -1), n(1, Sk, G, 64).expand(B, -1, -1, -1)
    else:
        q, k, v = n(B, Sq, H, 64), n(B, Sk, G, 64), n(B, Sk, G, 64)
    return q, k, v, n(B, Sq, H, 64)


def make_mask(kind, B, Sk, seed=1):
    g = torch.Generator().manual_seed(seed)
    m = torch.ones(B, Sk, dtype=torch.uint8)
    if kind == "none":
        return None
    if kind == "prefix":
        for b in range(B):
            m[b, int(torch.randint(1, Sk + 1, (1,), generator=g)):] = 0
    elif kind == "holes":
        m = (torch.rand(B, Sk, generator=g) < 0.6).to(torch.uint8) * 3
    elif kind == "empty":
        m[0] = 0
    elif kind == "blocks":  # whole blocks without a key, at the start and inside
        m[:, : min(70, Sk - 1)] = 0
        m[:, 128:200] = 0
        m[:, 256:320] = 0
    elif kind == "last":
        m[:] = 0
        m[:, Sk - 1] = 1
    return m.cuda()


def run(dtype, B, H, G, Sq, Sk, mask="none", causal=False, q_pos=None, relpos=None, layout="plain",
        scale=0.125, backward=True, garbage=False, seed=0):
    q, k, v, do = make(dtype, B, H, G, Sq, Sk, seed, layout)
    m = make_mask(mask, B, Sk)
    qp = None if q_pos is None else torch.tensor(q_pos, dtype=torch.int32).cuda()
    rp = table = None
    if relpos:
        rp = P.RelPos(*relpos)
        table = torch.randn(relpos[0], H, generator=torch.Generator().manual_seed(9)).cuda()
    if garbage:  # NaN and infinities in what the mask hides
        assert m is not None
        hide = (m == 0)[:, :, None, None]
        k, v = torch.where(hide, float("nan"), k), torch.where(hide, float("-inf"), v)
    kw = dict(scale=scale, causal=causal, q_pos=qp, table=table)
    want = reference(q, k, v, mask=m, relpos=relpos, dout=do if backward else None, **kw)
    out, lse = P.attn_forward(q, k, v, key_mask=m, relpos=rp, **kw)
    got = {"out": out, "lse": lse}
    if backward:
        got["dq"], got["dk"], got["dv"], dt = P.attn_backward(q, k, v, out, lse, do, key_mask=m,
                                                              relpos=rp, **kw)
        if relpos:
            got["dtable"] = dt
    torch.cuda.synchronize()
    ratio = {n: check(n, got[n], want[n]) for n in want}
    print({n: round(r, 3) for n, r in ratio.items()}, flush=True)
    return got


SIZES = [(1, 1), (1, 63), (2, 64), (31, 65), (32, 32), (33, 1), (64, 128), (77, 201), (128, 45),
         (129, 127), (130, 300), (257, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sq,sk", SIZES)
def test_lengths(dtype, sq, sk):
    run(dtype, 2, 2, 2, sq, sk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["prefix", "holes", "empty", "blocks", "last"])
@pytest.mark.parametrize("garbage", [False, True])
def test_masks(dtype, mask, garbage):
    run(dtype, 3, 2, 1, 70, 330, mask=mask, garbage=garbage)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["packed", "heads_first", "shared"])
@pytest.mark.parametrize("sq,sk", [(65, 65), (40, 150)])
def test_layouts(dtype, layout, sq, sk):
    run(dtype, 2, 4, 4, sq, sk, layout=layout, mask="holes")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(4, 1), (6, 2), (3, 3), (8, 4)])
def test_shared_key_heads(dtype, heads, kv):
    run(dtype, 2, heads, kv, 70, 150, mask="prefix")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sq,sk,q_pos", [(130, 130, None), (1, 200, [199, 3]), (5, 77, [0, 72]),
                                         (64, 40, [0, -30]), (33, 129, [-40, 500]),
                                         (200, 70, [-5, 10]), (3, 66, [2 ** 31 - 1, -2 ** 31])])
def test_causal(dtype, sq, sk, q_pos):
    run(dtype, 2, 2, 1, sq, sk, causal=True, q_pos=q_pos)
    run(dtype, 2, 2, 2, sq, sk, causal=True, q_pos=q_pos, mask="holes", garbage=True)


RELPOS = [(32, 128, True), (32, 128, False), (4, 5, True), (2, 3, False), (64, 512, True),
          (256, 2048, False), (10, 20, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("relpos", RELPOS)
def test_relpos(dtype, relpos):
    run(dtype, 2, 2, 2, 150, 150, relpos=relpos, causal=not relpos[2], layout="packed")
    run(dtype, 2, 4, 2, 70, 333, relpos=relpos, mask="prefix", q_pos=[100, -7])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["holes", "empty", "blocks", "last"])
def test_relpos_masks(dtype, mask):
    run(dtype, 2, 2, 1, 200, 330, relpos=(32, 128, True), mask=mask, garbage=True)
    run(dtype, 2, 2, 2, 130, 257, relpos=(16, 40, False), mask=mask, causal=True, q_pos=[120, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_relpos_beyond_every_key(dtype):
    run(dtype, 2, 2, 2, 40, 100, relpos=(32, 128, True), q_pos=[2 ** 31 - 1, -2 ** 31])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sq,sk,heads,kv", [(1, 1, 1, 1), (1, 77, 12, 12), (1, 700, 8, 2),
                                            (2, 1000, 4, 4), (4, 513, 8, 1), (1, 4500, 2, 2),
                                            (3, 2049, 16, 4), (1, 300, 64, 1)])
@pytest.mark.parametrize("relpos", [None, (32, 128, False)])
def test_tokens(dtype, sq, sk, heads, kv, relpos):
    pos = [sk - sq, max(0, sk // 3)]
    run(dtype, 2, heads, kv, sq, sk, causal=relpos is not None, relpos=relpos, q_pos=pos,
        backward=False, layout="packed")
    run(dtype, 2, heads, kv, sq, sk, mask="prefix", garbage=True, relpos=relpos, q_pos=pos,
        backward=False)
    run(dtype, 2, heads, kv, sq, sk, mask="empty", relpos=relpos, backward=False)


# (more tiles than the kernel for few queries takes, fewer work-groups than CUs: fp32
# wavefronts share their queries, and their keys)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 16, 8, 300, 130), (3, 12, 12, 257, 64), (9, 8, 8, 130, 33)])
@pytest.mark.parametrize("mask,garbage", [("none", False), ("empty", True), ("blocks", True),
                                          ("last", False), ("holes", True)])
@pytest.mark.parametrize("causal,relpos", [(False, None), (True, (32, 128, False)),
                                           (False, (16, 40, True))])
def test_shared_work(dtype, shape, mask, garbage, causal, relpos):
    run(dtype, *shape, mask=mask, garbage=garbage, causal=causal, relpos=relpos)


# (more splits of the keys than are joined at once)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,Sq,Sk", [(1, 1, 1, 1, 20000), (1, 2, 1, 2, 33000)])
@pytest.mark.parametrize("mask", ["none", "last", "holes"])
def test_tokens_over_long_caches(dtype, B, H, G, Sq, Sk, mask):
    run(dtype, B, H, G, Sq, Sk, mask=mask, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,Sq,Sk", [(1, 2, 1, 150000, 5), (1, 2, 1, 5, 150000)])
@pytest.mark.parametrize("causal,q_pos,relpos", [(False, None, None), (False, [40], (32, 128, True)),
                                                 (True, [149990], (32, 128, False))])
def test_one_long_side(dtype, B, H, G, Sq, Sk, causal, q_pos, relpos):
    run(dtype, B, H, G, Sq, Sk, causal=causal, q_pos=q_pos, relpos=relpos)


# (the heads of a key head go to several work-groups, beside those of dQ)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 8, 1, 20, 60), (3, 8, 2, 70, 130), (1, 16, 2, 40, 90),
                                   (2, 12, 2, 129, 33)])
@pytest.mark.parametrize("mask,garbage", [("none", False), ("empty", True), ("holes", True),
                                          ("last", False)])
@pytest.mark.parametrize("causal,q_pos", [(False, None), (True, [7, -3, 40])])
@pytest.mark.parametrize("relpos", [None, (8, 20, True)])
def test_shared_key_heads_of_few_queries(dtype, shape, mask, garbage, causal, q_pos, relpos):
    run(dtype, *shape, mask=mask, garbage=garbage, causal=causal,
        q_pos=None if q_pos is None else q_pos[:shape[0]], relpos=relpos)


# (each block to a work-group of its own, beside those of dQ)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 6, 3, 130, 128), (2, 4, 4, 200, 200), (3, 2, 1, 129, 300),
                                   (1, 3, 1, 20, 70), (2, 3, 3, 300, 90)])
@pytest.mark.parametrize("mask,garbage", [("none", False), ("empty", True), ("blocks", True)])
@pytest.mark.parametrize("causal,relpos", [(False, None), (True, None), (False, (32, 128, True)),
                                           (True, (32, 128, False))])
def test_two_or_three_blocks_of_queries(dtype, shape, mask, garbage, causal, relpos):
    run(dtype, *shape, mask=mask, garbage=garbage, causal=causal, relpos=relpos)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_queries_no_keys_no_batch(dtype):
    rp, dt = P.RelPos(8, 20), DT[dtype]
    for B, Sq, Sk in [(2, 0, 70), (2, 70, 0), (0, 5, 5), (2, 0, 0)]:
        q, k = torch.randn(B, Sq, 2, 64).to(dt).cuda(), torch.randn(B, Sk, 2, 64).to(dt).cuda()
        table = torch.randn(8, 2).cuda()
        out, lse = P.attn_forward(q, k, k.clone(), relpos=rp, table=table)
        grads = P.attn_backward(q, k, k.clone(), out, lse, torch.ones_like(q), relpos=rp,
                                table=table)
        assert not out.any() and torch.isneginf(lse).all()
        assert all(not g.any() for g in grads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    """Scores of hundreds: one key takes all, nothing overflows."""
    run(dtype, 1, 2, 2, 40, 200, scale=8.0)
    run(dtype, 1, 2, 2, 2, 200, scale=8.0, backward=False)


def test_gradients_against_differences():
    """Directional derivatives of <out, dout>, fp32 operands, central differences of
    the operator itself in steps where rounding (2^-24 of values near 1, over the
    step) and the third derivative (step squared) are both below the tolerance."""
    rp = P.RelPos(32, 128)
    q, k, v, do = make("f32", 2, 4, 2, 60, 90, seed=3)
    m = make_mask("holes", 2, 90)
    table = torch.randn(32, 4, generator=torch.Generator().manual_seed(2)).cuda()
    kw = dict(key_mask=m, relpos=rp)
    out, lse = P.attn_forward(q, k, v, table=table, **kw)
    grads = P.attn_backward(q, k, v, out, lse, do, table=table, **kw)
    args = [q, k, v, table]
    for i in range(4):
        d = torch.randn(args[i].shape, generator=torch.Generator().manual_seed(20 + i)).cuda()
        eps = 1e-2

        def value(sign):
            a = list(args)
            a[i] = a[i] + sign * eps * d
            o, _ = P.attn_forward(a[0], a[1], a[2], table=a[3], **kw)
            return float((o.double() * do.double()).sum())

        num = (value(1) - value(-1)) / (2 * eps)
        ana = float((grads[i].double() * d.double()).sum())
        size = float(grads[i].double().norm() * d.double().norm() / d.numel() ** 0.5)
        assert abs(num - ana) <= 2e-2 * max(abs(ana), size), (i, num, ana, size)


def test_same_bits_every_time():
    rp = P.RelPos(32, 128)
    q, k, v, do = make("bf16", 3, 8, 4, 300, 300, seed=5)
    m = make_mask("prefix", 3, 300)
    table = torch.randn(32, 8).cuda()
    runs = []
    for _ in range(3):
        out, lse = P.attn_forward(q, k, v, key_mask=m, relpos=rp, table=table)
        runs.append((out, lse) + P.attn_backward(q, k, v, out, lse, do, key_mask=m, relpos=rp,
                                                 table=table))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
