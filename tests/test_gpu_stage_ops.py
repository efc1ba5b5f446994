"""Stages that call the newer operators: rotary positions in the self attention, against torch's
float64 autograd of the same layers written out (tolerances as test_gpu_stage_attn.py), and AdamW
over a stage's own parameters."""
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import EPS, adamw64, frequencies, rotate, within
from paper_2202_11836_amd import PARAM_NAMES, Stage, StageError
from test_gpu_stage_attn import DT, bucket, close, ffn_half, ln, load, mask_of, params_of, rand

pytestmark = pytest.mark.gpu


def attn_half(x, p, H, rot=None, mask=None, table=None, relpos=None):
    """LN(x + W_o attention + b_o) with turned queries and keys."""
    B, S, h = x.shape
    q, k, v = (x @ p["W_qkv"].T + p["b_qkv"]).reshape(B, S, 3, H, 64).unbind(2)
    if rot is not None:
        n = rot.rot_dim // 2
        a = torch.arange(S, dtype=torch.float64)[:, None] * torch.tensor(frequencies(rot.rot_dim)).double()
        c, s = (rot.amplitude * f(a)[None, :, None] for f in (torch.cos, torch.sin))

        def turn(t):
            i0, i1 = (slice(0, n), slice(n, 2 * n)) if rot.layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
            y0, y1 = t[..., i0] * c - t[..., i1] * s, t[..., i0] * s + t[..., i1] * c
            y = torch.cat([y0, y1], -1) if rot.layout == "half" else torch.stack([y0, y1], -1).flatten(-2)
            return torch.cat([y, t[..., 2 * n:]], -1)

        q, k = turn(q), turn(k)
    sc = q.transpose(1, 2) @ k.transpose(1, 2).transpose(-1, -2) / 8.0
    if table is not None:
        ids = torch.tensor([[bucket(j - i, *relpos) for j in range(S)] for i in range(S)])
        sc = sc + table[ids].permute(2, 0, 1)
    see = torch.ones(B, S, dtype=torch.bool) if mask is None else mask != 0
    sc = sc.masked_fill(~see[:, None, None, :], -1e300)
    e = torch.exp(sc - sc.amax(-1, keepdim=True)) * see[:, None, None, :]
    pr = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
    c = (pr @ v.transpose(1, 2)).transpose(1, 2).reshape(B, S, h)
    return ln(x + c @ p["W_o"].T + p["b_o"], p["g1"], p["be1"])


def grads_close(st, layer, p, dtype, names=PARAM_NAMES):
    for n in names:
        close((layer, n), st.grad(layer, PARAM_NAMES.index(n)), p[n].grad, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,h,f,B,S,mask,rot,buckets", [
    (2, 128, 256, 2, 48, "prefix", dict(), None), (1, 256, 512, 3, 77, "holes", dict(rot_dim=32, layout="interleaved"), None),
    (2, 64, 128, 2, 150, "none", dict(rot_dim=20), (32, 128)), (1, 128, 256, 2, 33, "empty", dict(amplitude=1.5), None),
    (1, 64, 64, 1, 600, "prefix", dict(), None)])
def test_rotary_layers(dtype, L, h, f, B, S, mask, rot, buckets):
    H, rot = h // 64, P.Rotary(**rot)
    ps = [params_of(h, f, 7 + l, dtype) for l in range(L)]
    st = Stage(L, h, H, f, dtype=dtype)
    for l, p in enumerate(ps):
        load(st, l, p)
    table = relpos = None
    if buckets:
        relpos = (buckets[0], buckets[1], True)
        table = rand((buckets[0], H), 3, 0.7).double().requires_grad_()
        st.set_relpos(*buckets)
        st.relpos_table().copy_(table.detach())
    st.set_rotary(rot)
    x, dy = rand((B, S, h), 1).to(DT[dtype]), rand((B, S, h), 2).to(DT[dtype])
    m = mask_of(B, S, mask)
    y = st.forward(x.cuda(), None if m is None else m.cuda())
    dx = st.backward(dy.cuda())
    xr = x.double().requires_grad_()
    t = xr
    for p in ps:
        t = ffn_half(attn_half(t, p, H, rot, m, table, relpos), p)
    (t * dy.double()).sum().backward()
    close("y", y, t, dtype, True)
    close("dx", dx, xr.grad, dtype)
    for l, p in enumerate(ps):
        grads_close(st, l, p, dtype)
    if buckets:
        close("table", st.relpos_grad(), table.grad, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotary_halves_chain(dtype):
    """An attention half and a feed-forward half as stages of their own, by their units."""
    h, f, B, S, rot = 128, 192, 2, 45, P.Rotary(layout="interleaved")
    p = params_of(h, f, 5, dtype)
    a = Stage(None, h, 2, f, dtype=dtype, first_unit=0, n_units=1)
    b = Stage(None, h, 2, f, dtype=dtype, first_unit=1, n_units=1)
    load(a, 0, p, PARAM_NAMES[:6])
    load(b, 0, p, PARAM_NAMES[6:])
    a.set_rotary(rot)
    with pytest.raises(StageError) as e:
        b.set_rotary(rot)
    assert e.value.status == 1 and "attention half" in str(e.value)
    x, dy = rand((B, S, h), 1).to(DT[dtype]).cuda(), rand((B, S, h), 2).to(DT[dtype]).cuda()
    y = b.forward(a.forward(x))
    dx = a.backward(b.backward(dy))
    xr = x.cpu().double().requires_grad_()
    t = ffn_half(attn_half(xr, p, 2, rot), p)
    (t * dy.cpu().double()).sum().backward()
    close("y", y, t, dtype, True)
    close("dx", dx, xr.grad, dtype)
    grads_close(a, 0, p, dtype, PARAM_NAMES[:6])
    grads_close(b, 0, p, dtype, PARAM_NAMES[6:])


@pytest.mark.parametrize("dtype,h,B,S", [("f32", 128, 2, 48), ("bf16", 128, 2, 48), ("bf16", 1024, 32, 512)])
def test_rotary_on_and_off(dtype, h, B, S):
    """Taken out again the stage is as before, bit for bit; frequencies of 0 turn nothing; the
    saved Q and K are the turned ones; a context from before is not taken."""
    st = Stage(1, h, h // 64, 2 * h, seed=3, dtype=dtype)
    x, dy = rand((B, S, h), 1).to(DT[dtype]).cuda(), rand((B, S, h), 2).to(DT[dtype]).cuda()

    def run():
        y = st.forward(x)
        qkv = st.saved(0, 1, B * S).view(B, S, 3, h // 64, 64)
        return [y, st.backward(dy)] + [st.grad(0, i) for i in range(12)], qkv

    plain, qkv = run()
    rot = P.Rotary(40)
    st.forward(x)
    st.set_rotary(rot)
    with pytest.raises(StageError) as e:
        st.backward(dy)
    assert e.value.status == 2
    turned, after = run()
    assert not torch.equal(plain[0], turned[0])
    for i in range(2):
        want, tol = rotate(qkv[:, :, i], frequencies(40), "half", None)
        within(i, after[:, :, i], want, tol)
    assert torch.equal(after[:, :, 2], qkv[:, :, 2])
    st.set_rotary(P.Rotary(8, freqs=[0.0] * 4))
    still, _ = run()
    # (the same context; the column sums of db_qkv go in another order)
    for i, (a, b) in enumerate(zip(plain, still)):
        if i == 2 + PARAM_NAMES.index("b_qkv"):
            assert ((a - b).norm() / a.norm()).item() < 1e-2 if dtype == "bf16" else (a - b).abs().max() < 1e-4 * a.abs().max()
        else:
            assert torch.equal(a, b), i
    st.set_rotary(None)
    again, _ = run()
    assert all(torch.equal(a, b) for a, b in zip(plain, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotary_noalloc_and_graph(dtype):
    """stage_backward_noalloc makes the same bits; a captured step follows its input."""
    h, B, S = 128, 3, 70
    st = Stage(2, h, 2, 256, seed=4, dtype=dtype)
    st.set_rotary(P.Rotary())
    x, dy = rand((B, S, h), 1).to(DT[dtype]).cuda(), rand((B, S, h), 2).to(DT[dtype]).cuda()
    st.forward(x)
    dx = st.backward(dy)
    grads = [st.grad(l, i) for l in range(2) for i in range(12)]
    st.forward(x)
    other = st.backward_noalloc(dy, torch.empty_like(dy))
    assert torch.equal(dx, other)
    assert all(torch.equal(a, st.grad(l, i)) for a, (l, i) in zip(grads, [(l, i) for l in range(2) for i in range(12)]))
    y, out = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        st.forward(x, out=y)
        st.backward(dy, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        st.forward(x, out=y)
        st.backward(dy, out=out)
    for i in range(3):
        x.copy_(rand((B, S, h), 10 + i))
        g.replay()
        torch.cuda.synchronize()
        got = y.clone(), out.clone()
        want = st.forward(x), st.backward(dy)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rotary_refusals():
    st = Stage(None, 64, 1, 64, first_unit=0, n_units=1, dtype="f32")
    st.set_rotary(P.Rotary())
    x = torch.zeros(1, 4, 64, device="cuda")
    with pytest.raises(StageError) as e:
        st.forward_cross(x, x.clone())
    assert e.value.status == 1 and "rotary" in str(e.value)
    bad = P.Rotary().c
    bad.rot_dim = 3
    with pytest.raises(StageError) as e:
        P.stage_set_rotary(st.handle, bad)
    assert e.value.status == 1 and "rot_dim" in str(e.value)
    st.forward(x)  # (as before)
    st.set_rotary(None)
    st.forward_cross(x, x.clone())
    st.forward(torch.zeros(0, 4, 64, device="cuda"))


# ---------------------------------------------------------------------------
# AdamW of a stage
# ---------------------------------------------------------------------------
LR, BETAS = 1e-3, (0.9, 0.99)


def values(st, opt):
    return [st.param(l, PARAM_NAMES.index(n)) if l is not None else st.relpos_table().clone() for l, n in opt.names]


@pytest.mark.parametrize("dtype,units,relpos", [("f32", (0, 4), False), ("bf16", (0, 4), True), ("bf16", (1, 2), False),
                                                ("f32", (0, 1), True), ("bf16", (3, 1), False)])
def test_adamw_of_a_stage(dtype, units, relpos):
    """Steps behind backward passes: each parameter as the formula makes it of the gradient that the
    stage gives, the next forward with the new ones."""
    h = 128
    st = Stage(None, h, 2, 192, seed=2, dtype=dtype, first_unit=units[0], n_units=units[1])
    if relpos:
        st.set_relpos(32, 128)
    opt = st.adamw(weight_decay=0.1, betas=BETAS)
    held = sum(1 for l in range(st.L) for w in range(12) if st.handle and P.binding.load_library().stage_tensor_bytes(st.handle, 0, l, w))
    assert len(opt.params) == held + relpos and len(set(opt.names)) == len(opt.names)
    x, dy = (rand((2, 40, h), i).to(DT[dtype]).cuda() for i in (1, 2))
    m = [torch.zeros(p.shape, dtype=torch.float64, device="cuda") for p in opt.params]
    v, most = ([t.clone() for t in m] for _ in range(2))
    w = [t.float().clone() for t in opt.params]
    outs = []
    for t in range(1, 4):
        outs.append(st.forward(x))
        st.backward(dy)
        before = values(st, opt)
        assert all(torch.equal(a, b) for a, b in zip(before, opt.params))
        opt.step(LR)
        for i, (l, n) in enumerate(opt.names):
            g = st.grad(l, PARAM_NAMES.index(n)) if l is not None else st.relpos_grad()
            decay = 0.1 if n[0] == "W" else 0.0
            # m in fp32 is off by 3 EPS a step of the size of its terms, 0.9 |m| and 0.1 |g|, which
            # may be far above m where they cancel: with `most` the sum of the terms' sizes over the
            # steps, by 3 EPS most (v's terms do not cancel: 4 t EPS of itself, half of that in its
            # root).  So the update is off by 3 EPS of what it were with most in m's place.
            most[i] = BETAS[0] * most[i] + (1 - BETAS[0]) * g.double().abs()
            w64, m[i], v[i], up = adamw64(w[i], g, m[i], v[i], t, LR, BETAS, 1e-8, decay)
            wide = LR * most[i] / (1 - BETAS[0] ** t) / ((v[i] / (1 - BETAS[1] ** t)).sqrt() + 1e-8)
            tol = 4 * EPS * w[i].double().abs() + (32 + 8 * t) * EPS * up.abs() + 3 * t * EPS * wide
            got = opt.state["master"][i] if opt.state["master"][i] is not None else opt.params[i]
            within((t, l, n), got, w64, tol)
            w[i] = got.clone()
            if opt.state["master"][i] is not None:
                assert torch.equal(opt.params[i], got.bfloat16())
        assert not any(torch.equal(a, b) for (a, b, n) in zip(before, values(st, opt), opt.names) if n[1] == "b_1")
    assert not torch.equal(outs[0], outs[1]) and not torch.equal(outs[1], outs[2])


def test_adamw_of_a_stage_in_a_graph():
    """forward, backward and step captured together, replayed, against eager ones of a second stage."""
    h, x, dy = 128, rand((2, 40, 128), 1).to(torch.bfloat16).cuda(), rand((2, 40, 128), 2).to(torch.bfloat16).cuda()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    stages = [Stage(2, h, 2, 256, seed=2) for _ in range(2)]
    opts = [st.adamw(state_bits=8) for st in stages]
    for st in stages:
        st.set_rotary(P.Rotary())
    for st, opt in zip(stages, opts):
        st.forward(x, out=y)
        st.backward(dy, out=dx)
        opt.step(LR, max_norm=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        stages[0].forward(x, out=y)
        stages[0].backward(dy, out=dx)
        opts[0].step(LR, max_norm=0.1)
    for i in range(3):
        x.copy_(rand((2, 40, 128), 20 + i))
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, stages[1].forward(x))
        stages[1].backward(dy)
        opts[1].step(LR, max_norm=0.1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(opts[0].params, opts[1].params)), i
        assert torch.equal(opts[0].norm, opts[1].norm)


def test_adamw_of_a_stage_that_is_gone():
    st = Stage(1, 64, 1, 64, seed=2)
    opt = st.adamw()
    st.set_relpos(32, 128)
    with pytest.raises(StageError) as e:
        opt.step(LR)
    assert e.value.status == 2 and "table" in str(e.value)
    opt = st.adamw()
    assert opt.names[-1] == (None, "relpos_table")
    x = torch.ones(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    st.forward(x)
    st.backward(x)
    opt.step(LR)
    st.close()
    with pytest.raises(StageError) as e:
        opt.step(LR)
    assert e.value.status == 2 and "closed" in str(e.value)
    with pytest.raises(StageError) as e:
        st.adamw()
    assert e.value.status == 2 and "closed" in str(e.value)


def test_master_copies_of_a_stage_that_is_gone():
    st = Stage(1, 64, 1, 64, seed=2)
    opt = st.adamw()
    st.set_param(0, 0, st.param(0, 0) + 1)
    opt.reset_master()
    assert all(w is None or torch.equal(w, p.float()) for p, w in zip(opt.params, opt.state["master"]))
    st.close()
    with pytest.raises(StageError) as e:
        opt.reset_master()
    assert e.value.status == 2 and "closed" in str(e.value)
