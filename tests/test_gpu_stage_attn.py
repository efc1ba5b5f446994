"""Stages that call the attention operators: encoder layers with a relative position
bias, an attention half as cross attention over an encoder's output, and both in a
row, against torch's float64 autograd of the same layers written out.

Tolerances are the stage's own (fp32: largest difference 1e-4 of the largest value;
bf16: relative 2-norm 1e-2, outputs of a LayerNorm 2e-2 or a bf16 step)."""
import math

import pytest
import torch

import paper_2202_11836_amd as P
from _attn_ref import bucket
from paper_2202_11836_amd import PARAM_NAMES, Stage, StageError

pytestmark = pytest.mark.gpu
ATTN = PARAM_NAMES[:6]
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(shape, seed, std=1.0, mean=0.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std + mean


def params_of(h, f, seed, dtype):
    """One layer's parameters, float64 CPU, matrices rounded to the stage's type."""
    shapes = {"W_qkv": (3 * h, h), "b_qkv": (3 * h,), "W_o": (h, h), "W_1": (f, h), "b_1": (f,),
              "W_2": (h, f)}
    p = {}
    for i, n in enumerate(PARAM_NAMES):
        shape = shapes.get(n, (h,))
        if n[0] == "W":
            w = rand(shape, 100 * seed + i, 0.06).to(DT[dtype]).float()
        else:
            w = rand(shape, 100 * seed + i, 0.1, 1.0 if n[0] == "g" else 0.0)
        p[n] = w.double().requires_grad_()
    return p


def load(st, layer, p, names=PARAM_NAMES):
    for n in names:
        st.set_param(layer, PARAM_NAMES.index(n), p[n].detach().float().cuda())


def ln(z, g, b):
    mu = z.mean(-1, keepdim=True)
    return g * (z - mu) / torch.sqrt(((z - mu) ** 2).mean(-1, keepdim=True) + 1e-12) + b


def attn_half(x, mem, p, H, mask=None, table=None, relpos=None):
    """LN(x + W_o attention + b_o); mem is x for self attention."""
    B, S, h = x.shape
    M = mem.shape[1]
    w, b = p["W_qkv"], p["b_qkv"]

    def heads(t, lo):
        return (t @ w[lo:lo + h].T + b[lo:lo + h]).reshape(B, -1, H, 64).transpose(1, 2)

    q, k, v = heads(x, 0), heads(mem, h), heads(mem, 2 * h)
    s = q @ k.transpose(-1, -2) / 8.0
    if table is not None:
        ids = torch.tensor([[bucket(j - i, *relpos) for j in range(M)] for i in range(S)])
        s = s + table[ids].permute(2, 0, 1)
    see = torch.ones(B, M, dtype=torch.bool) if mask is None else mask != 0
    s = s.masked_fill(~see[:, None, None, :], -1e300)
    e = torch.exp(s - s.amax(-1, keepdim=True)) * see[:, None, None, :] if M else s
    pr = e / e.sum(-1, keepdim=True).clamp(min=1e-300) if M else s
    c = (pr @ v).transpose(1, 2).reshape(B, S, h)
    return ln(x + c @ p["W_o"].T + p["b_o"], p["g1"], p["be1"])


def ffn_half(x, p):
    u = x @ p["W_1"].T + p["b_1"]
    g = u * 0.5 * torch.erfc(-u / math.sqrt(2.0))
    return ln(x + g @ p["W_2"].T + p["b_2"], p["g2"], p["be2"])


def close(name, got, want, dtype, out=False):
    got, want = got.detach().cpu().double(), want.detach().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert torch.isfinite(got).all(), name
    d = got - want
    if dtype == "f32":
        err = float(d.abs().max() / want.abs().max().clamp(min=1e-30)) if want.numel() else 0.0
        assert err <= 1e-4, (name, err)
    elif out:
        step = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=1e-30))) - 7)
        err = float((d.abs() / torch.clamp(step, min=2e-2)).max())
        assert err <= 1.0, (name, err)
    else:
        err = float(d.norm() / want.norm().clamp(min=1e-30))
        assert err <= 1e-2, (name, err)
    return err


def check_grads(st, layer, p, dtype, names=PARAM_NAMES):
    h = st.hidden
    worst = 0.0
    for n in names:
        got, want = st.grad(layer, PARAM_NAMES.index(n)).cpu(), p[n].grad
        if n == "b_qkv":  # a key bias shifts whole rows of scores: no gradient
            tol = (1e-4 if dtype == "f32" else 1e-2) * float(want[:h].norm())
            assert float(got[h:2 * h].double().norm()) <= tol
            got, want = torch.cat([got[:h], got[2 * h:]]), torch.cat([want[:h], want[2 * h:]])
        worst = max(worst, close(n, got, want, dtype))
    return worst


def mask_of(B, S, kind):
    m = torch.ones(B, S, dtype=torch.uint8)
    if kind == "none":
        return None
    for b in range(B):
        m[b, S - (7 * b + 3) % S:] = 0
    if kind == "holes":
        m[:, ::5] = 0
    if kind == "empty":
        m[B - 1] = 0
    return m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,h,f,B,S,mask,buckets", [(2, 128, 256, 2, 48, "prefix", (32, 128)),
                                                    (1, 256, 512, 3, 77, "holes", (16, 20)),
                                                    (2, 64, 128, 2, 150, "none", (64, 256)),
                                                    (1, 128, 256, 2, 33, "empty", (8, 64)),
                                                    (1, 64, 64, 1, 600, "prefix", (32, 128))])
def test_relpos_layers(dtype, L, h, f, B, S, mask, buckets):
    H, relpos = h // 64, (buckets[0], buckets[1], True)
    ps = [params_of(h, f, 7 + l, dtype) for l in range(L)]
    table = rand((buckets[0], H), 3, 0.7).double().requires_grad_()
    st = Stage(L, h, H, f, dtype=dtype)
    for l, p in enumerate(ps):
        load(st, l, p)
    st.set_relpos(*buckets)
    assert not st.relpos_table().any() and st.relpos_table().shape == (buckets[0], H)
    st.relpos_table().copy_(table.detach())
    x, dy = rand((B, S, h), 1).to(DT[dtype]), rand((B, S, h), 2).to(DT[dtype])
    m = mask_of(B, S, mask)
    y = st.forward(x.cuda(), None if m is None else m.cuda())
    dx = st.backward(dy.cuda())
    xr = x.double().requires_grad_()
    z = xr
    for p in ps:
        z = ffn_half(attn_half(z, z, p, H, m, table, relpos), p)
    z.backward(dy.double())
    close("y", y, z, dtype, out=L == 1)
    close("dx", dx, xr.grad, dtype)
    for l, p in enumerate(ps):
        check_grads(st, l, p, dtype)
    close("table", st.relpos_grad(), table.grad, dtype)
    # again, and through the backward that may not allocate: the same bits
    keep = [st.grad(l, i) for l in range(L) for i in range(12)] + [st.relpos_grad().clone(), dx, y]
    y2 = st.forward(x.cuda(), None if m is None else m.cuda())
    dx2 = st.backward_noalloc(dy.cuda(), torch.empty_like(dx))
    again = [st.grad(l, i) for l in range(L) for i in range(12)] + [st.relpos_grad().clone(), dx2, y2]
    assert all(torch.equal(a, b) for a, b in zip(keep, again))
    st.close()


def test_relpos_of_zeros_and_without():
    """A table of zeros computes the same function as no bias; taking the bias out
    gives the earlier bits back."""
    st = Stage(2, 128, 2, 256, seed=4, dtype="f32")
    x, dy = rand((2, 60, 128), 5).cuda(), rand((2, 60, 128), 6).cuda()
    m = mask_of(2, 60, "prefix").cuda()
    y0, dx0 = st.forward(x, m), st.backward(dy)
    bytes0 = st.device_bytes()
    st.set_relpos(32)
    y1, dx1 = st.forward(x, m), st.backward(dy)
    assert float((y1 - y0).abs().max()) <= 1e-4 * float(y0.abs().max())
    assert float((dx1 - dx0).abs().max()) <= 1e-4 * float(dx0.abs().max())
    assert st.device_bytes() > bytes0
    st.set_relpos(0)
    assert torch.equal(st.forward(x, m), y0) and torch.equal(st.backward(dy), dx0)
    assert st.device_bytes() == bytes0
    with pytest.raises(StageError) as e:
        st.relpos_table()
    assert e.value.status == 2
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_relpos_half_layers(dtype):
    """Units [1, 4): a feed-forward half, a layer's attention and feed-forward halves:
    the table's gradient comes from the one attention half."""
    h, f, H, B, S = 128, 256, 2, 2, 40
    ps = [params_of(h, f, 21 + l, dtype) for l in range(2)]
    st = Stage(None, h, H, f, dtype=dtype, first_unit=1, n_units=3)
    load(st, 0, ps[0], PARAM_NAMES[6:])
    load(st, 1, ps[1])
    st.set_relpos(16, 30)
    table = rand((16, H), 8).double().requires_grad_()
    st.relpos_table().copy_(table.detach())
    x, dy = rand((B, S, h), 9).to(DT[dtype]), rand((B, S, h), 10).to(DT[dtype])
    st.forward(x.cuda())
    dx = st.backward(dy.cuda())
    xr = x.double().requires_grad_()
    z = ffn_half(xr, ps[0])
    ffn_half(attn_half(z, z, ps[1], H, None, table, (16, 30, True)), ps[1]).backward(dy.double())
    close("dx", dx, xr.grad, dtype)
    close("table", st.relpos_grad(), table.grad, dtype)
    check_grads(st, 1, ps[1], dtype)
    # an empty batch has zero gradients, the table's too
    e = torch.empty((0, S, h), dtype=DT[dtype], device="cuda")
    st.forward(e)
    st.backward(e)
    assert not st.relpos_grad().any() and not st.grad(1, 0).any()
    st.close()


CROSS = [(2, 48, 77, 128, "prefix"), (3, 1, 50, 64, "holes"), (2, 130, 33, 128, "empty"),
         (1, 300, 1, 64, "none"), (4, 20, 260, 256, "none"), (2, 5, 0, 64, "none")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,M,h,mask", CROSS)
def test_cross(dtype, B, S, M, h, mask):
    H = h // 64
    p = params_of(h, 64, 31, dtype)
    st = Stage(None, h, H, 64, dtype=dtype, first_unit=0, n_units=1)
    load(st, 0, p, ATTN)
    x, mem = rand((B, S, h), 11).to(DT[dtype]), rand((B, M, h), 12).to(DT[dtype])
    dy = rand((B, S, h), 13).to(DT[dtype])
    m = mask_of(B, M, mask) if M else None
    y = st.forward_cross(x.cuda(), mem.cuda(), None if m is None else m.cuda())
    dx, dmem = st.backward_cross(dy.cuda())
    xr, mr = x.double().requires_grad_(), mem.double().requires_grad_()
    z = attn_half(xr, mr, p, H, m)
    z.backward(dy.double())
    close("y", y, z, dtype, out=True)
    close("dx", dx, xr.grad, dtype)
    if M > 1:
        close("dmem", dmem, mr.grad, dtype)
        check_grads(st, 0, p, dtype, ATTN)
    elif M == 1:  # one key: its probability is 1 and no score has a gradient
        close("dmem", dmem, mr.grad, dtype)
        close("W_v", st.grad(0, 0).cpu()[2 * h:], p["W_qkv"].grad[2 * h:], dtype)
        size = float(p["W_qkv"].grad[2 * h:].abs().max())
        assert float(st.grad(0, 0)[:2 * h].abs().max()) <= 1e-2 * size
    else:
        assert not st.grad(0, 0)[h:].any() and not st.grad(0, 1)[h:].any()
    if m is not None:
        assert not dmem[(m == 0).cuda()].any()
    # the same bits again, and after a self-attention pass in between
    keep = [st.grad(0, i) for i in range(6)] + [dx, dmem, y]
    st.forward(x.cuda())
    with pytest.raises(StageError) as e:
        st.backward_cross(dy.cuda())
    assert e.value.status == 2
    y2 = st.forward_cross(x.cuda(), mem.cuda(), None if m is None else m.cuda())
    for call in (lambda: st.backward(dy.cuda()),
                 lambda: st.backward_noalloc(dy.cuda(), torch.empty_like(dx))):
        with pytest.raises(StageError) as e:
            call()
        assert e.value.status == 2
    dx2, dmem2 = st.backward_cross(dy.cuda())
    again = [st.grad(0, i) for i in range(6)] + [dx2, dmem2, y2]
    assert all(torch.equal(a, b) for a, b in zip(keep, again))
    with pytest.raises(StageError) as e:
        st.backward_cross(dy.cuda())
    assert e.value.status == 2
    st.close()


def test_cross_sizes_in_turn():
    """One stage over batches that grow and shrink, against fresh stages."""
    p = params_of(128, 64, 41, "bf16")
    st = Stage(None, 128, 2, 64, dtype="bf16", first_unit=0, n_units=1)
    load(st, 0, p, ATTN)
    for i, (B, S, M) in enumerate([(2, 30, 40), (3, 100, 10), (1, 7, 900), (2, 30, 40), (0, 5, 5),
                                   (2, 0, 6), (8, 64, 64)]):
        x, mem = rand((B, S, 128), 50 + i).bfloat16().cuda(), rand((B, M, 128), 60 + i).bfloat16().cuda()
        y, (dx, dm) = st.forward_cross(x, mem), st.backward_cross(torch.ones_like(x))
        one = Stage(None, 128, 2, 64, dtype="bf16", first_unit=0, n_units=1)
        load(one, 0, p, ATTN)
        yo, (dxo, dmo) = one.forward_cross(x, mem), one.backward_cross(torch.ones_like(x))
        assert torch.equal(y, yo) and torch.equal(dx, dxo) and torch.equal(dm, dmo)
        assert all(torch.equal(st.grad(0, j), one.grad(0, j)) for j in range(6))
        if B * S == 0:
            assert not dm.any() and not st.grad(0, 0).any()
        one.close()
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_encoder_with_bias_then_cross(dtype):
    """An encoder stage with the bias, its output the memory of a cross-attention half,
    and the gradient back through both."""
    h, f, H, B, S, T = 128, 256, 2, 2, 70, 25
    ps = [params_of(h, f, 51 + l, dtype) for l in range(3)]
    enc = Stage(2, h, H, f, dtype=dtype)
    for l in range(2):
        load(enc, l, ps[l])
    enc.set_relpos(32, 128)
    table = rand((32, H), 14, 0.5).double().requires_grad_()
    enc.relpos_table().copy_(table.detach())
    dec = Stage(None, h, H, f, dtype=dtype, first_unit=4, n_units=1)
    load(dec, 0, ps[2], ATTN)
    src, tgt = rand((B, S, h), 15).to(DT[dtype]), rand((B, T, h), 16).to(DT[dtype])
    dy, m = rand((B, T, h), 17).to(DT[dtype]), mask_of(B, S, "prefix")
    mem = enc.forward(src.cuda(), m.cuda())
    y = dec.forward_cross(tgt.cuda(), mem, m.cuda())
    dtgt, dmem = dec.backward_cross(dy.cuda())
    dsrc = enc.backward(dmem)
    sr, tr = src.double().requires_grad_(), tgt.double().requires_grad_()
    z = sr
    for l in range(2):
        z = ffn_half(attn_half(z, z, ps[l], H, m, table, (32, 128, True)), ps[l])
    out = attn_half(tr, z, ps[2], H, m)
    out.backward(dy.double())
    close("y", y, out, dtype)
    close("dtgt", dtgt, tr.grad, dtype)
    # bf16: the gradient crosses the boundary rounded, and the bias's gradient is the
    # end of three layers of bf16 tensors: the deep stages' bound of two layers' worth
    for name, a, b in (("dsrc", dsrc, sr.grad), ("table", enc.relpos_grad(), table.grad)):
        err = float((a.cpu().double() - b).norm() / b.norm())
        assert err <= (1e-4 if dtype == "f32" else 2e-2), (name, err)
    enc.close()
    dec.close()


def test_cross_in_a_graph():
    """A captured cross step replayed on new inputs, with eager work in between."""
    p = params_of(128, 64, 61, "bf16")
    st = Stage(None, 128, 2, 64, dtype="bf16", first_unit=0, n_units=1)
    load(st, 0, p, ATTN)
    x, mem = torch.zeros(2, 30, 128).bfloat16().cuda(), torch.zeros(2, 45, 128).bfloat16().cuda()
    m, dy = mask_of(2, 45, "prefix").cuda(), torch.zeros_like(x)
    y, dx, dm = torch.empty_like(x), torch.empty_like(x), torch.empty_like(mem)

    def step():
        st.forward_cross(x, mem, m, out=y)
        st.backward_cross(dy, out=dx, out_memory=dm)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    ref = Stage(None, 128, 2, 64, dtype="bf16", first_unit=0, n_units=1)
    load(ref, 0, p, ATTN)
    for i in range(3):
        for t, k in ((x, 0), (mem, 1), (dy, 2)):
            t.copy_(rand(tuple(t.shape), 70 + 3 * i + k))
        g.replay()
        torch.cuda.synchronize()
        yr, (dxr, dmr) = ref.forward_cross(x, mem, m), ref.backward_cross(dy)
        assert torch.equal(y, yr) and torch.equal(dx, dxr) and torch.equal(dm, dmr)
        assert all(torch.equal(st.grad(0, j), ref.grad(0, j)) for j in range(6))
    del g
    st.close()
    ref.close()


def test_refusals():
    layer = Stage(1, 128, 2, 256, dtype="f32")
    half = Stage(None, 128, 2, 256, dtype="f32", first_unit=0, n_units=1)
    ffn = Stage(None, 128, 2, 256, dtype="f32", first_unit=1, n_units=1)
    x = torch.zeros(1, 4, 128, device="cuda")

    def refused(call, status=1):
        with pytest.raises(StageError) as e:
            call()
        assert e.value.status == status and str(e.value)

    refused(lambda: layer.forward_cross(x, x.clone()))
    refused(lambda: ffn.forward_cross(x, x.clone()))
    refused(lambda: ffn.set_relpos(32))
    for b, d in ((33, 128), (2, 128), (32, 8), (32, 5000), (-1, 128)):
        refused(lambda: layer.set_relpos(b, d))
    refused(lambda: half.forward_cross(x, x.clone(), out=x))
    refused(lambda: half.backward_cross(x), 2)
    refused(lambda: P.stage_forward_cross(half.handle, x, None, None, 1, 4, 4, torch.empty_like(x)))
    refused(lambda: P.stage_forward_cross(half.handle, x, x, None, 1, 4, -1, torch.empty_like(x)))
    half.set_relpos(32)
    refused(lambda: half.forward_cross(x, x.clone()))
    for s in (layer, half, ffn):
        s.close()
