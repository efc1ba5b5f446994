"""AdamW over many tensors: fp32 states against float64 within bounds derived from the formulas,
8-bit states bit for bit (every operation on them is rounded by itself), sizes around vectors,
blocks and chunks, alignment, clipping, steps that are skipped, graphs and streams, and the
optimizer of a stage."""
import math

import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import DT, EPS, adamw64, decode, encode, rand, random_bits, states32, within

pytestmark = pytest.mark.gpu
LR, EPS_A, BETAS = 1e-2, 1e-8, (0.9, 0.999)
SIZES = [1, 7, 8, 9, 255, 256, 257, 2047, 2048, 2049, 0, 100003]


def grads_of(sizes, dtype, seed):
    """Gradients whose size differs by a factor of 100 within a tensor, zeros among them."""
    out = []
    for i, n in enumerate(sizes):
        g = rand((n,), 100 * seed + i) * torch.exp(rand((n,), 100 * seed + i + 50) * 1.5) * 1e-2
        g[::11] = 0
        out.append(g.to(DT[dtype]))
    return out


class Tensors:
    """Parameters, gradients and an optimizer over them."""

    def __init__(self, sizes, dtype="f32", grad="f32", bits=32, master=True, decay=0.1, **kw):
        self.params = [rand((n,), 7 + i, dtype) for i, n in enumerate(sizes)]
        self.grads = grads_of(sizes, grad, 1)
        self.kw = dict(betas=BETAS, eps=EPS_A, weight_decay=decay, state_bits=bits, master=master, **kw)
        self.opt = P.AdamW(self.params, self.grads, **self.kw)

    def new_grads(self, seed):
        for g, h in zip(self.grads, grads_of([g.numel() for g in self.grads], "f32", seed)):
            g.copy_(h)

    def all(self):
        s = self.opt.state
        return [t.view(torch.uint8) if t.element_size() == 1 else t for t in
                self.params + [t for n in self.opt.LISTS for t in s[n] if t is not None] + [s["steps"]]]


def copies(ts):
    return [t.clone() for t in ts]


def expected(w, g, m, v, t, bits, dtype, master, decay, clip=None, lr=LR, lr_scale=1.0):
    """What a step makes of one tensor: (w64, the largest part of its error, m, v as they are
    kept, the parameter if it has to be equal)."""
    if bits == 8:
        m, v = decode(*m), decode(*v)
    m32, v32 = states32(g, m, v, BETAS, clip)
    w64, _, _, up = adamw64(w, g, m, v, t, lr * lr_scale, BETAS, EPS_A, decay,
                            1.0 if clip is None else float(clip))
    tol = 4 * EPS * w.double().abs() + 32 * EPS * up.abs() + EPS * w64.abs()
    r = random_bits(w.numel(), t)
    if bits == 8:
        m32, v32 = encode(m32, "e4m3", r & 0xFFFF), encode(v32, "e5m2", r >> 16)
    return w64, tol, m32, v32, r


def check_step(x, t, decay, clip=None, lr=LR, lr_scale=1.0):
    """One step of x.opt against what it has to be."""
    s, opt = x.opt.state, x.opt
    before = [(p.clone(), *[None if s[n][i] is None else s[n][i].clone() for n in opt.LISTS])
              for i, p in enumerate(x.params)]
    opt.step(torch.tensor([lr], device="cuda") if t % 2 else lr, max_norm=None if clip is None else 1.0)
    assert s["steps"].item() == t
    for i, (p, (p0, m, v, ms, vs, w)) in enumerate(zip(x.params, before)):
        if not p.numel():
            continue
        bits = opt.state_bits[i]
        start = (p0 if w is None else w).float()
        w64, tol, m2, v2, r = expected(start, x.grads[i], (m, ms) if bits == 8 else m,
                                       (v, vs) if bits == 8 else v, t, bits, p.dtype, w is not None, decay,
                                       clip, lr, lr_scale)
        if bits == 8:
            for name, (codes, scale) in (("exp_avg", m2), ("exp_avg_sq", v2)):
                assert torch.equal(s[name][i].view(torch.uint8), codes), (name, i)
                torch.testing.assert_close(s[name + "_scale"][i], scale, rtol=0, atol=0, equal_nan=True)
        else:
            assert torch.equal(s["exp_avg"][i], m2) and torch.equal(s["exp_avg_sq"][i], v2), i
        if p.dtype == torch.float32:
            within(("param", i), p, w64, tol)
        elif w is not None:
            within(("master", i), s["master"][i], w64, tol)
            assert torch.equal(p, s["master"][i].bfloat16())
        else:
            # the upper neighbour where the bits say so: that rounding never falls where its
            # argument grows, so p lies between what the ends of w's range become
            lo, hi = (((y.float().view(torch.int32).long() + (r >> 16)) >> 16).to(torch.int16).view(torch.bfloat16)
                      for y in (w64 - tol, w64 + tol))
            assert ((lo <= p) & (p <= hi)).all(), i
            assert (lo == hi).float().mean() > 0.99  # (mostly a single value)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad,master", [("f32", "f32", True), ("f32", "bf16", True), ("bf16", "f32", True),
                                               ("bf16", "bf16", True), ("bf16", "bf16", False),
                                               ("bf16", "f32", False)])
def test_steps(dtype, grad, master, bits):
    x = Tensors(SIZES, dtype, grad, bits, master)
    for t in range(1, 5):
        x.new_grads(t)
        check_step(x, t, 0.1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "bf16")])
def test_ends(dtype, grad, bits):
    """Each number of elements behind the last whole eight, in the first block, in a later one and just
    behind a chunk, between NaN that no result shows."""
    sizes = [b + r for b in (0, 8, 248, 1024, 2040, 2048) for r in range(1, 8)]
    x = Tensors(sizes, dtype, grad, bits, master=False)
    big = [[torch.full((n + 16,), float("nan"), device="cuda", dtype=t.dtype) for n, t in zip(sizes, ts)]
           for ts in (x.params, x.grads)]
    for views, ts in zip(big, (x.params, x.grads)):
        for i, t in enumerate(list(ts)):
            views[i][8:-8] = t
            ts[i] = views[i][8:-8]
    x.opt = P.AdamW(x.params, x.grads, **x.kw)
    for t in range(1, 3):
        check_step(x, t, 0.1)
    for t in big[0] + big[1]:
        assert t[:8].isnan().all() and t[-8:].isnan().all()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_any_number_of_chunks(bits):
    """The number of steps is raised once, by however many work-groups there are."""
    for n in (1, 2, 31, 32, 33, 63, 64, 65, 100, 511, 512, 513, 1023, 1024, 1025, 2000):
        p, g = torch.ones(2048 * n, device="cuda").bfloat16(), torch.ones(2048 * n, device="cuda").bfloat16()
        opt = P.AdamW([p], [g], weight_decay=0.0, state_bits=bits, master=False)
        for t in range(1, 5):
            opt.step(0.0)
            assert opt.state["steps"].item() == t, n
        # 1 - 0.9^4 = 0.3439.  fp32: three roundings a step, 12 * 2^-24 * 0.35 in all.  8 bits: each
        # step adds at most 2^-3 of the value to 0.9 of the error, 0.0125, 0.037, 0.071, 0.115.
        m = opt.state["exp_avg"][0].float().view(-1, 256)
        if bits == 8:
            m = m * opt.state["exp_avg_scale"][0][:, None]
        assert (m - (1 - 0.9 ** 4)).abs().max() < (0.115 if bits == 8 else 2.6e-7), n
        assert (p == 1).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_late_steps(bits):
    """A step counter beyond 32 bits: no bias is left, the bits' step wraps."""
    x = Tensors([5000], bits=bits)
    for t in (1000, 2 ** 32 + 5):
        x.opt.state["steps"].fill_(t - 1)
        check_step(x, t, 0.1)


@pytest.mark.parametrize("bits", [32, 8])
def test_any_alignment(bits):
    """Tensors that begin at any element; what lies around them stays."""
    n, every = 3000, {}

    def part(dtype, at, size=n):
        t = torch.zeros(size + 64, device="cuda").to(dtype)
        t.view(torch.uint8).fill_(0x31)
        every[len(every)] = (t, at, size, t.clone())
        return t[at:at + size]

    params, grads, state = [], [], {k: [] for k in P.AdamW.LISTS}
    for i, dtype in enumerate((torch.float32, torch.bfloat16, torch.bfloat16)):
        params.append(part(dtype, 1 + i).copy_(rand((n,), i)))
        grads.append(part((torch.bfloat16, torch.float32)[i % 2], 3).copy_(rand((n,), 9 + i)))
        eight = bits == 8
        state["exp_avg"].append(part(torch.float8_e4m3fn if eight else torch.float32, 1 + i).zero_())
        state["exp_avg_sq"].append(part(torch.float8_e5m2 if eight else torch.float32, 5).zero_())
        for k in ("exp_avg_scale", "exp_avg_sq_scale"):
            state[k].append(part(torch.float32, 3, 12).zero_() if eight else None)
        state["master"].append(part(torch.float32, 1).copy_(params[-1]) if i == 1 else None)
    state["steps"] = torch.zeros(1, dtype=torch.int64, device="cuda")
    x = Tensors([])
    x.params, x.grads = params, grads
    x.opt = P.AdamW(params, grads, betas=BETAS, eps=EPS_A, weight_decay=0.1, state_bits=bits, state=state)
    for t in (1, 2):
        check_step(x, t, 0.1)
    for t, at, size, was in every.values():
        t, was = t.view(torch.uint8), was.view(torch.uint8)
        e = t.numel() // (size + 64)
        assert torch.equal(t[:at * e], was[:at * e]) and torch.equal(t[(at + size) * e:], was[(at + size) * e:])


def test_settings_of_each_tensor():
    """Decay, rate and bits by tensor."""
    x = Tensors([4000, 4000, 3000, 300])
    decay, scale, bits = [0.0, 0.1, 0.2, 0.0], [1.0, 0.5, 0.0, 2.0], [32, 8, 8, 32]
    x.opt = P.AdamW(x.params, x.grads, betas=BETAS, eps=EPS_A, weight_decay=decay, lr_scale=scale, state_bits=bits)
    start = copies(x.params)
    x.opt.step(LR)
    assert torch.equal(x.params[2], start[2])
    for i in range(4):
        zero = torch.zeros_like(start[i])
        w64, _, _, up = adamw64(start[i], x.grads[i], zero, zero, 1, LR * scale[i], BETAS, EPS_A, decay[i])
        within(i, x.params[i], w64, 5 * EPS * start[i].double().abs() + 32 * EPS * up.abs())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_clipping(grad, bits):
    """Gradients in whole numbers of 2^-10, so that the sum of their squares is exact: the
    clipped step bit for bit, the norm, and one that needs no clipping."""
    x = Tensors(SIZES, grad=grad, bits=bits)
    for t in (1, 2):
        total = 0.0
        for i, g in enumerate(x.grads):
            gen = torch.Generator(device="cuda").manual_seed(10 * t + i)
            g.copy_(torch.randint(-9, 10, g.shape, generator=gen, device="cuda") * (2.0 ** -10 if t == 1 else 2.0 ** -14))
            total += g.double().square().sum().item()
        norm = math.sqrt(total)
        assert (norm > 1.0) == (t == 1)
        check_step(x, t, 0.1, clip=torch.tensor(min(1.0, 1.0 / norm), dtype=torch.float32).cuda())
        assert abs(x.opt.norm.item() - norm) <= EPS * norm
    # more gradients than the norm has work-groups, and ones whose squares fp32 cannot hold
    y = Tensors([3_000_000], grad="f32")
    y.grads[0].fill_(1e25)
    before = copies(y.params)
    assert abs(y.opt.step(LR, max_norm=1.0).item() / (1e25 * math.sqrt(3e6)) - 1) < 4 * EPS
    assert y.opt.state["steps"].item() == 1 and y.params[0].isfinite().all() and not torch.equal(before[0], y.params[0])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_not_finite(value, bits):
    """With clipping the step changes nothing; without, it reaches its own element, or its block."""
    x = Tensors([3000, 1000], bits=bits)
    x.opt.step(LR)
    x.grads[0][700] = value
    before = copies(x.all())
    norm = x.opt.step(LR, max_norm=1.0)
    assert not math.isfinite(norm.item()) and all(torch.equal(a, b) for a, b in zip(before, x.all()))
    y = Tensors([3000, 1000], bits=bits)
    y.opt.step(LR)
    y.opt.step(LR)
    x.opt.step(LR)
    s, z = x.opt.state, y.opt.state
    hit = torch.zeros(3000, dtype=torch.bool, device="cuda")
    hit[700] = True
    assert not x.params[0][700].isfinite() and torch.equal(x.params[0][~hit], y.params[0][~hit])
    assert torch.equal(x.params[1], y.params[1])
    if bits == 8:
        hit[512:768] = True
        m = decode(s["exp_avg"][0], s["exp_avg_scale"][0])
        assert m[hit].isnan().all() and torch.equal(m[~hit], decode(z["exp_avg"][0], z["exp_avg_scale"][0])[~hit])
    else:
        assert not s["exp_avg"][0][700].isfinite()
        assert torch.equal(s["exp_avg"][0][~hit], z["exp_avg"][0][~hit])


def test_small_blocks_and_zeros():
    """Blocks of zeros, of values whose squares are below fp32's normal range, of one large value
    among small ones, and of values whose squares are beyond fp32 (which count as not finite)."""
    x = Tensors([2048], bits=8)
    g = x.grads[0]
    g.fill_(0.0)
    g[256:512] = 1e-30
    g[512:768] = 1e-8
    g[600] = 1.0
    g[768:1024] = -1e30
    for t in range(1, 4):
        check_step(x, t, 0.1)
    s = x.opt.state
    v = decode(s["exp_avg_sq"][0], s["exp_avg_sq_scale"][0])
    assert (v[:512] == 0).all() and (v[512:768] > 0).all() and v[768:1024].isnan().all()
    live = torch.ones(2048, dtype=torch.bool, device="cuda")
    live[768:1024] = False
    assert x.params[0][live].isfinite().all()


def test_states_in_8_bits_follow_those_in_32():
    """100 steps over gradients that shrink by 10 on the way: on average over the elements the
    8-bit second moment is the fp32 one.  Each step rounds at random with the right mean: an
    element is off by at most some 50%, 65536 of them on average by 0.5 / 256 = 0.2%, 5 times
    that is 1%; codes that may not become 0 raise the small ones' by less than 2^-16 of the
    block's largest."""
    n = 1 << 16
    size = torch.exp(rand((n // 256, 1), 3)).expand(-1, 256).reshape(-1)
    opts = []
    for bits in (8, 32):
        p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        opts.append((P.AdamW([p], [g], betas=(0.9, 0.98), state_bits=bits, weight_decay=0.0), p, g))
    for t in range(100):
        h = rand((n,), 100 + t) * size * (1.0 if t < 50 else 0.1)
        for o, _, g in opts:
            g.copy_(h)
            o.step(1e-3)
    s = opts[0][0].state
    v8, v32 = decode(s["exp_avg_sq"][0], s["exp_avg_sq_scale"][0]).double(), opts[1][0].state["exp_avg_sq"][0].double()
    assert abs((v8 / v32).mean().item() - 1) < 0.01
    m8, m32 = decode(s["exp_avg"][0], s["exp_avg_scale"][0]).double(), opts[1][0].state["exp_avg"][0].double()
    # (of m too: its mean error, in units of the elements' own size)
    assert abs(((m8 - m32) / m32.abs().mean()).mean().item()) < 0.01
    a, b = opts[0][1].double(), opts[1][1].double()
    assert (a * b).sum() / (a.norm() * b.norm()) > 0.99


def test_weights_without_master_move():
    """Updates of a fiftieth of a bf16 step: rounded to nearest none would be left."""
    n = 1 << 16
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, dtype=torch.bfloat16, device="cuda")
    o = P.AdamW([p], [g], weight_decay=0.0, master=False)
    lr, steps = 2.0 ** -8 / 50, 40  # (below 1 a bf16 step is 2^-8)
    for _ in range(steps):
        o.step(lr)
    # each element's move is a sum of draws with the right mean: 65536 of them, 5 deviations
    moved = 1.0 - p.double().mean().item()
    assert abs(moved - lr * steps) < 5 * 2.0 ** -8 * math.sqrt(steps / 50) / 256


def test_state_goes_on():
    """Another optimizer on the first one's states (copied) makes the same steps."""
    for bits in (32, 8):
        x = Tensors([5000, 77], "bf16", "bf16", bits)
        x.opt.step(LR)
        s = {n: [None if t is None else t.clone() for t in x.opt.state[n]] for n in x.opt.LISTS}
        s["steps"] = x.opt.state["steps"].clone()
        y = Tensors([5000, 77], "bf16", "bf16", bits)
        for a, b in zip(y.params, x.params):
            a.copy_(b)
        y.opt = P.AdamW(y.params, y.grads, state=s, **y.kw)
        for _ in range(2):
            x.opt.step(LR)
            y.opt.step(LR)
        assert all(torch.equal(a, b) for a, b in zip(x.all(), y.all()))


def test_states_taken_out_of_the_lists():
    """The memory of states stays the optimizer's when another tensor takes their place in a list."""
    x, y = Tensors([50000]), Tensors([50000])
    x.opt.state["exp_avg"][0] = x.params[0] = torch.zeros(1, device="cuda")
    held = x.opt._held
    junk = [torch.full((50000,), float("nan"), device="cuda") for _ in range(20)]
    for _ in range(2):
        x.opt.step(LR)
        y.opt.step(LR)
    assert torch.equal(held[0], y.params[0]) and all(j.isnan().all() for j in junk)


def test_reset_master():
    x = Tensors([300], "bf16")
    x.params[0].copy_(rand((300,), 50))
    x.opt.reset_master()
    assert torch.equal(x.opt.state["master"][0], x.params[0].float())


def test_leaves_of_a_graph():
    """Parameters that autograd knows: the states are none of its."""
    p = rand((5, 300), 1, "bf16").requires_grad_()
    g = torch.zeros_like(p)
    opt = P.AdamW([p], [g], state_bits=8)
    (p.float() ** 2).sum().backward()
    g.copy_(p.grad)
    opt.step(LR)
    opt.reset_master()
    for n in opt.LISTS:
        t = opt.state[n][0]
        assert t is not None and t.grad_fn is None and not t.requires_grad, n
    assert p.is_leaf and p.requires_grad and torch.equal(opt.state["master"][0], p.detach().float())


def test_nothing_to_update():
    for sizes in ([], [0, 0]):
        x = Tensors(sizes)
        x.opt.step(LR)
        assert x.opt.step(LR, max_norm=1.0).item() == 0.0 and x.opt.state["steps"].item() == 2


def test_many_tensors():
    """800 tensors of 1 to 3000 elements, in one call; the rows in between of no other."""
    sizes = [1 + (i * 7919) % 3000 for i in range(800)]
    x = Tensors(sizes)
    before = copies(x.params)
    x.opt.step(LR)
    for i in range(0, 800, 37):
        z = torch.zeros_like(before[i])
        w64, _, _, up = adamw64(before[i], x.grads[i], z, z, 1, LR, BETAS, EPS_A, 0.1)
        within(i, x.params[i], w64, 5 * EPS * before[i].double().abs() + 32 * EPS * up.abs())


def test_more_than_2_31_elements():
    n = (1 << 31) + 300
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = rand((600,), 1, "bf16")
    g[-600:], g[:600] = tail, tail
    o = P.AdamW([p], [g], betas=BETAS, state_bits=8, master=False, weight_decay=0.0)
    norm = o.step(LR, max_norm=1e9).item()
    assert abs(norm / (2 * tail.double().square().sum()).sqrt().item() - 1) < 4 * EPS
    s = o.state
    z = torch.zeros(600, device="cuda")
    m32, v32 = states32(tail, z, z, BETAS)
    at = n - 600
    first = at // 256
    m = decode(s["exp_avg"][0][first * 256:], s["exp_avg_scale"][0][first:])[at - first * 256:]
    assert ((m - m32).abs() <= m32.abs() * 0.125 + 2.0 ** -9 / 448 * m32.abs().max()).all()
    assert (p[600:-600] == 0).all() and torch.equal(p[-600:] == 0, p[:600] == 0)
    live = tail != 0
    assert ((p[-600:][live].float() + LR * tail[live].sign()).abs() < LR * 0.02).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_graph(bits):
    """A captured step counts on, follows its rate and its gradients, and clips."""
    x, y = (Tensors([5000, 260, 9], "bf16", "f32", bits) for _ in range(2))
    lr = torch.full((1,), 1e-3, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x.opt.step(lr, max_norm=0.5)
    y.opt.step(lr, max_norm=0.5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        norm = x.opt.step(lr, max_norm=0.5)
    for i in range(1, 5):
        lr.fill_(1e-3 * i)
        x.new_grads(i)
        y.new_grads(i)
        g.replay()
        torch.cuda.synchronize()
        want = y.opt.step(lr, max_norm=0.5)
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(x.all(), y.all())), i
    assert x.opt.state["steps"].item() == 5


def test_two_at_once():
    """Optimizers of their own on streams of their own."""
    xs = [Tensors([400000, 3000], "bf16", "bf16", bits) for bits in (32, 8, 32)]
    streams = [torch.cuda.Stream() for _ in xs]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for x, st in zip(xs, streams):
            with torch.cuda.stream(st):
                x.opt.step(LR, max_norm=1.0)
    torch.cuda.synchronize()
    for x, bits in zip(xs, (32, 8, 32)):
        y = Tensors([400000, 3000], "bf16", "bf16", bits)
        for _ in range(5):
            y.opt.step(LR, max_norm=1.0)
        assert all(torch.equal(a, b) for a, b in zip(x.all(), y.all()))


def test_tensors_that_move():
    """A step is refused while a tensor is of other memory, and nothing is written to the old or the new."""
    x = Tensors([5000, 300], "bf16", "bf16", 8)
    x.opt.step(LR)
    for t in (x.params[0], x.grads[1], x.opt.state["master"][1], x.opt.state["exp_avg_scale"][0]):
        back, other = t.data, torch.full_like(t, 3)
        t.data = other
        was = copies(x.opt._held)
        with pytest.raises(P.StageError) as e:
            x.opt.step(LR, max_norm=1.0)
        assert e.value.status == 1 and "other memory" in str(e.value)
        torch.cuda.synchronize()
        assert (other == 3).all()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(was, x.opt._held))
        t.data = back
    net = torch.nn.Linear(64, 32, device="cuda")
    for p in net.parameters():
        p.grad = torch.ones_like(p)
    opt = P.AdamW(list(net.parameters()), [p.grad for p in net.parameters()])
    opt.step(LR)
    net.bfloat16()
    with pytest.raises(P.StageError) as e:
        opt.step(LR)
    assert "params[0]" in str(e.value)
    assert opt.state["steps"].item() == 1
    y = Tensors([5000, 300], "bf16", "bf16", 8)
    for _ in range(2):
        y.opt.step(LR)
    x.opt.step(LR)
    assert all(torch.equal(a, b) for a, b in zip(x.all(), y.all()))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("pattern", [0x7fc00000, 0x7fffffff, -1, 0x7f800001, 0x7fbfffff, -0x400001])
def test_any_nan_reaches_its_weight(pattern, master, bits):
    """NaN with any low bits, in a gradient or in a weight, whatever the draw of its rounding."""
    n = 20000
    x, y = (Tensors([n], "bf16", "f32", bits, master) for _ in range(2))
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    hit[3::37] = True
    x.grads[0].view(torch.int32)[hit] = pattern
    x.opt.step(LR)
    y.opt.step(LR)
    assert x.params[0][hit].isnan().all() and torch.equal(x.params[0][~hit], y.params[0][~hit])
    if bits == 32:
        assert x.opt.state["exp_avg"][0][hit].isnan().all() and x.opt.state["exp_avg_sq"][0][hit].isnan().all()
    z = Tensors([n], "bf16", "f32", bits, False)
    z.params[0].view(torch.int16)[hit] = pattern >> 16 | 0x40  # (a bf16 NaN, quiet)
    z.opt.step(LR)
    assert z.params[0][hit].isnan().all() and z.params[0][~hit].isfinite().all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-30, 1e-20, 1e-17, 1e-8])
def test_subnormal_second_moments(eps, dtype, bits):
    """Gradients whose squares are subnormal in v: it is held as such and has its root, so an eps far
    below that root leaves updates of the usual size.  Weights of 0, so that w is the update: off
    by the roundings of rate, rate m, root, its product, the sum, reciprocal (1 EPS each, root and
    reciprocal 2) and the last product, 9 EPS, from the states in fp32 as they are defined."""
    n = 4096
    w = torch.zeros(n, device="cuda")
    p = w.to(DT[dtype])
    g = rand((n,), 1) * torch.exp(rand((n,), 2) * 2.0) * 1e-18
    g[::5] = 0
    g[1::64] = 3e-12  # (among others whose squares are not subnormal)
    zero = torch.zeros(n, device="cuda")
    opt = P.AdamW([p], [g], betas=BETAS, eps=eps, weight_decay=0.0, state_bits=bits)
    opt.step(LR)
    m, v = states32(g, zero, zero, BETAS)
    tiny = (v > 0) & (v < torch.finfo(torch.float32).tiny)
    assert tiny.sum() > n // 4 and (v >= torch.finfo(torch.float32).tiny).any()
    if bits == 32:
        assert torch.equal(opt.state["exp_avg"][0], m) and torch.equal(opt.state["exp_avg_sq"][0], v)
    up = LR * (m.double() / (1 - BETAS[0])) / ((v.double() / (1 - BETAS[1])).sqrt() + eps)
    got = p if dtype == "f32" else opt.state["master"][0]
    within("w", got, -up, 9 * EPS * up.abs() + 2.0 ** -149)
    if eps == 1e-30:
        # An update of the size of the rate.  Of v above 2^-140 the rounding, 2^-150, is 2^-10 of it and 2^-11
        # of its root, g^2's before, 2^-150 of some 1000 v, less; eps is below 1e-10 of sqrt(v / 0.001).  (For
        # 1e-20 it is up to 0.4 of that root, which the bound above has and this one had not.)
        some = tiny & (v > 2.0 ** -140)
        assert some.any() and ((got[some].abs() - LR).abs() < LR * 2.0 ** -9).all()


def test_tensors_that_are_copied_when_written():
    """Their own memory comes with the address that the handle takes, and is where they stay."""
    x, y = Tensors([3000, 100]), Tensors([3000, 100])
    was = copies(x.params)
    x.opt = P.AdamW([torch._lazy_clone(p) for p in x.params], [torch._lazy_clone(g) for g in x.grads], **x.kw)
    for _ in range(2):
        x.opt.step(LR)
        y.opt.step(LR)
    assert all(torch.equal(a, b) for a, b in zip(x.opt.params, y.params))
    assert all(torch.equal(a, b) for a, b in zip(x.params, was))


def test_tensors_of_inference():
    """Parameters and states made in inference mode."""
    with torch.inference_mode():
        x = Tensors([3000], "bf16")
        x.opt.step(LR)
    y = Tensors([3000], "bf16")
    y.opt.step(LR)
    x.opt.step(LR)
    y.opt.step(LR)
    assert torch.equal(x.params[0], y.params[0])
