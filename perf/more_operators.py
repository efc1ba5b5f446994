"""Timed cases of the operators around a stage in a training step: the AdamW update
of many tensors at once, layer norm with its gradients, and rotary positions of
queries and keys.

A case is one call of `AdamW.step`, of `layer_norm_forward` (step: and
`layer_norm_backward`) or of `rotary_forward` (step: and `rotary_backward`) on tensors
that a program holds at that point.

Fields of a case, by its "op":
  adamw   the tensors of `layers` encoder layers (`hidden`, `ffn`): matrices of
          `dtype` ("bf16": with fp32 master copies, "bf16_alone": without; "f32"),
          vectors fp32; grad: type of the matrices' gradients; bits: 32 or 8, the
          matrices' states; clip: gradients clipped by their global norm
  norm    rows [batch, seq] of `width` values; residual: a tensor is added first;
          mode "forward" or "step"
  rotary  q [batch, seq, heads, 64], k with kv_heads; rot: values of a head that are
          rotated; layout "half" or "interleaved"; scaling "none", "linear", "base"
          or "parts" by `factor`; mode "token" (positions of their own, up to
          max_pos), "forward" or "step" (positions from 0)
"""
import math

import numpy as np
import torch

own = False
HEAD_DIM = 64
EPS_NORM = 1e-12
LR, BETAS, EPS_ADAM, DECAY, MAX_NORM = 1e-4, (0.9, 0.999), 1e-8, 0.01, 1.0
BLOCK = 256  # elements that share a scale of 8-bit states
ORIGINAL_LEN, LOW, HIGH, BASE = 2048, 1.0, 32.0, 10000.0


def _adamw(name, layers, hidden, ffn, dtype, grad="f32", bits=32, clip=False):
    return {"name": name, "op": "adamw", "layers": layers, "hidden": hidden, "ffn": ffn,
            "dtype": dtype, "grad": grad, "bits": bits, "clip": clip}


def _norm(name, mode, dtype, batch, seq, width, residual=False):
    return {"name": name, "op": "norm", "mode": mode, "dtype": dtype, "batch": batch, "seq": seq,
            "width": width, "residual": residual}


def _rotary(name, mode, dtype, batch, seq, heads, kv_heads, rot=64, layout="half", scaling="none",
            factor=1.0, max_pos=0):
    return {"name": name, "op": "rotary", "mode": mode, "dtype": dtype, "batch": batch, "seq": seq,
            "heads": heads, "kv_heads": kv_heads, "rot": rot, "layout": layout, "scaling": scaling,
            "factor": factor, "max_pos": max_pos}


def listed():
    return [
        # The weights of the tiny fp32 stage (width 128): latency.
        _adamw("adamw_tiny_f32", 2, 128, 512, "f32"),
        # A share of four layers of odd sizes, fp32 throughout, clipped.
        _adamw("adamw_odd_clip", 4, 321, 1283, "f32", clip=True),
        # Four layers of width 1024 with states in 8 bits, gradients in bf16.
        _adamw("adamw_large4_8bit", 4, 1024, 4096, "bf16", grad="bf16", bits=8),
        # The 40 layers of the depth sweep: 504 million weights, 15 GB, clipped.
        _adamw("adamw_deep40", 40, 1024, 4096, "bf16", clip=True),
        # One token of each of 8 sequences before the next stage.
        _norm("norm_tokens", "forward", "bf16", 8, 1, 1024),
        # The fp32 check of a step, odd sizes.
        _norm("norm_odd_f32_step", "step", "f32", 3, 77, 765),
        # The 32 x 512 batch between two layers, with its residual addition.
        _norm("norm_large_step", "step", "bf16", 32, 512, 1024, True),
        # Wide rows of a few long documents.
        _norm("norm_wide_step", "step", "bf16", 2, 2500, 5120),
        # A token for each of 32 sequences, each at its own position, four query
        # heads to a key head.
        _rotary("rotary_tokens", "token", "bf16", 32, 1, 16, 4, max_pos=8192),
        # The fp32 check of a step: pairs side by side, a part of the head, odd length.
        _rotary("rotary_odd_f32_step", "step", "f32", 3, 77, 12, 12, 20, "interleaved"),
        # One layer's queries and keys of the 32 x 512 batch.
        _rotary("rotary_large_step", "step", "bf16", 32, 512, 16, 16),
        # Documents 16 times as long as those trained on, half of each head.
        _rotary("rotary_long_forward", "forward", "bf16", 2, 32768, 16, 4, 32, "interleaved",
                "parts", 16.0),
    ]


def _sizes(c):
    """(numbers of elements of the matrices, of the vectors) of all layers."""
    h, f = c["hidden"], c["ffn"]
    return [3 * h * h, h * h, f * h, h * f] * c["layers"], [3 * h, h, h, h, f, h, h, h] * c["layers"]


def _esz(c, what="dtype"):
    return 4 if c[what] == "f32" else 2


def work(case):
    c = case
    if c["op"] == "adamw":
        mats, vecs = (float(sum(s)) for s in _sizes(c))
        state = 2 * 2 * (4 if c["bits"] == 32 else 1 + 4 / BLOCK)  # two states, read and written
        weight = {"f32": 8, "bf16": 8 + 2, "bf16_alone": 4}[c["dtype"]]
        return {"bytes": mats * (weight + _esz(c, "grad") + state) + vecs * 28,
                "flops": 20.0 * (mats + vecs)}
    if c["op"] == "norm":
        rows, n = c["batch"] * c["seq"], float(c["batch"] * c["seq"] * c["width"])
        # x, y (and the residual and the sum); step: their gradients too
        tensors = (4 if c["residual"] else 2) + ((3 if c["residual"] else 2) if c["mode"] == "step" else 0)
        return {"bytes": n * tensors * _esz(c) + rows * 8 + c["width"] * (16 if c["mode"] == "step" else 8),
                "flops": n * (20 if c["mode"] == "step" else 8)}
    n = float(c["batch"] * c["seq"] * (c["heads"] + c["kv_heads"]))
    times = 2 if c["mode"] == "step" else 1
    return {"bytes": times * n * 2 * HEAD_DIM * _esz(c), "flops": times * n * 3 * c["rot"]}


def draw(rng):
    """One more case: operators, types, modes and sizes over the ranges of the listed
    cases."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("adamw", "norm", "rotary"))
    most = max(work(c)["bytes"] for c in listed() if c["op"] == op)
    while True:
        if op == "adamw":
            bits = rng.choice((32, 8))
            dtype = rng.choice(("f32", "bf16", "bf16", "bf16_alone"))
            hidden = spread(64, 1500)
            c = _adamw("", spread(1, 40), hidden, spread(hidden, 4 * hidden), dtype,
                       "f32" if dtype == "f32" else rng.choice(("f32", "bf16")), bits,
                       bits == 32 and rng.random() < 0.5)
            # (8 bits: up to 100 million weights, whose plain form is the slowest)
            fits = bits == 32 or sum(_sizes(c)[0]) < 100e6
        elif op == "norm":
            mode, dtype = rng.choice(("forward", "step", "step")), rng.choice(("bf16", "bf16", "f32"))
            width = rng.choice((spread(64, 8192), 64 * spread(1, 128)))
            c = _norm("", mode, dtype, spread(1, 32), spread(1, 4096), width, rng.random() < 0.4)
            fits = True
        else:
            mode, dtype = rng.choice(("token", "forward", "step", "step")), rng.choice(("bf16", "bf16", "f32"))
            kv = rng.choice((1, 2, 4, 8, 12, 16))
            scaling = rng.choice(("none", "none", "linear", "base", "parts"))
            c = _rotary("", mode, dtype, spread(1, 32),
                        rng.choice((1, 1, 2, 4)) if mode == "token" else spread(2, 32768),
                        kv * rng.choice((1, 1, 2, 4)), kv, rng.choice((64, 64, 32, 16, 2 * rng.randint(2, 31))),
                        rng.choice(("half", "interleaved")), scaling,
                        1.0 if scaling == "none" else round(rng.uniform(1.5, 32.0), 2),
                        spread(32, 1 << 20) if mode == "token" else 0)
            fits = c["heads"] <= 64
        del c["name"]
        if fits and work(c)["bytes"] <= most:
            return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 4241)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _group(sizes, dtype, grad, bits, master, decay, g):
    """Tensors of these sizes, each of which begins a block of one memory a quantity, and
    their states after some steps: gradients whose size differs from block to block."""
    at = np.concatenate([[0], np.cumsum([-(-n // BLOCK) * BLOCK for n in sizes])]).astype(np.int64)
    blocks = int(at[-1]) // BLOCK
    ids = np.repeat(np.arange(len(sizes)), np.diff(at) // BLOCK)
    # of each block: the element of its tensor that it begins with
    first = torch.from_numpy(np.arange(blocks) * BLOCK - at[ids]).cuda()
    if len(set(sizes)) == 1 and sizes[0] % BLOCK == 0:
        live = None
    else:
        left = torch.from_numpy(np.array(sizes)[ids]).cuda() - first
        live = torch.arange(BLOCK, device="cuda")[None, :] < left[:, None]

    def values(t):
        return t if live is None else t.masked_fill_(~live, 0.0)

    size = torch.exp(_normal(g, (blocks, 1))) * 1e-3
    s = {"sizes": sizes, "at": at.tolist(), "decay": decay, "bits": bits, "first": first, "live": live}
    w = values(_normal(g, (blocks, BLOCK), 0.02))
    s["p"] = w.to(_type(dtype))
    s["master"] = w if master else None
    s["g"] = values(_normal(g, (blocks, BLOCK)) * size).to(_type(grad))
    m = values(_normal(g, (blocks, BLOCK)) * size * 0.3)
    v = values(torch.empty((blocks, BLOCK), device="cuda").uniform_(0.5, 1.5, generator=g) * size * size)
    s["m_scale"] = s["v_scale"] = None
    if bits == 8:
        half = torch.full_like(s["p"], 0x8000, dtype=torch.int32)
        m, s["m_scale"] = _to_e4m3(m, half)
        v, s["v_scale"] = _to_e5m2(v, half)
    s["m"], s["v"] = m, v
    return s


def _adamw_inputs(case, seed):
    c, g = case, _generator(seed)
    mats, vecs = _sizes(c)
    dtype = "f32" if c["dtype"] == "f32" else "bf16"
    groups = [_group(mats, dtype, c["grad"], c["bits"], c["dtype"] == "bf16", DECAY, g),
              _group(vecs, "f32", "f32", 32, False, 0.0, g)]
    steps = torch.full((1,), 20 + seed % 1000, dtype=torch.int64, device="cuda")
    return {"groups": groups, "steps": steps}


def _norm_inputs(case, seed):
    c, g = case, _generator(seed)
    shape, dt = (c["batch"], c["seq"], c["width"]), _type(c["dtype"])
    s = {"x": (_normal(g, shape) + 0.3).to(dt), "gamma": 1.0 + _normal(g, (c["width"],), 0.2),
         "beta": _normal(g, (c["width"],), 0.2), "residual": None, "dy": None, "dtotal": None}
    if c["residual"]:
        s["residual"] = _normal(g, shape).to(dt)
    if c["mode"] == "step":
        s["dy"] = _normal(g, shape).to(dt)
        if c["residual"]:
            s["dtotal"] = _normal(g, shape).to(dt)
    return s


def _rotary_inputs(case, seed):
    """q and k as parts of one projection, as a program has them."""
    c, g = case, _generator(seed)
    B, S, H, G = c["batch"], c["seq"], c["heads"], c["kv_heads"]

    def both():
        t = _normal(g, (B, S, H + 2 * G, HEAD_DIM)).to(_type(c["dtype"]))
        return t[:, :, :H], t[:, :, H:H + G]

    s = {"pos": None}
    s["q"], s["k"] = both()
    if c["mode"] == "token":
        pos = np.random.default_rng(seed).integers(0, max(c["max_pos"] - S, 1), size=B)
        s["pos"] = torch.from_numpy(pos.astype(np.int32)).cuda()
    if c["mode"] == "step":
        s["dq"], s["dk"] = both()
    return s


def _views(s, name):
    t = s[name].view(-1)
    return [t[a:a + n] for a, n in zip(s["at"], s["sizes"])]


def _scales(s, name):
    return [s[name][a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in zip(s["at"], s["sizes"])]


def _optimizer(s):
    """The optimizer that a program keeps: it updates the tensors it is given in place."""
    import paper_2202_11836_amd as P
    params, grads, decay, bits = [], [], [], []
    state = {n: [] for n in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "master")}
    for t in s["groups"]:
        n, eight = len(t["sizes"]), t["bits"] == 8
        params += _views(t, "p")
        grads += _views(t, "g")
        decay += [t["decay"]] * n
        bits += [t["bits"]] * n
        state["exp_avg"] += _views(t, "m")
        state["exp_avg_sq"] += _views(t, "v")
        state["exp_avg_scale"] += _scales(t, "m_scale") if eight else [None] * n
        state["exp_avg_sq_scale"] += _scales(t, "v_scale") if eight else [None] * n
        state["master"] += _views(t, "master") if t["master"] is not None else [None] * n
    state["steps"] = s["steps"]
    return P.AdamW(params, grads, betas=BETAS, eps=EPS_ADAM, weight_decay=decay, state_bits=bits,
                   state=state)


def prepare(case, seed):
    c = case
    if c["op"] == "adamw":
        s = _adamw_inputs(c, seed)
        if own:
            s["optimizer"] = _optimizer(s)
    elif c["op"] == "norm":
        s = _norm_inputs(c, seed)
        if own:
            s["out"] = {"out": torch.empty_like(s["x"])}
            if c["residual"]:
                s["out"]["total"] = torch.empty_like(s["x"])
            if c["mode"] == "step":
                s["grads"] = {"dx": torch.empty_like(s["x"]), "dgamma": torch.empty_like(s["gamma"]),
                              "dbeta": torch.empty_like(s["beta"])}
    else:
        s = _rotary_inputs(c, seed)
        if own:
            import paper_2202_11836_amd as P
            s["rotary"] = P.Rotary(c["rot"], BASE, layout=c["layout"],
                                   scaling=None if c["scaling"] == "none" else c["scaling"],
                                   factor=c["factor"], original_len=ORIGINAL_LEN, low=LOW, high=HIGH,
                                   amplitude=_amplitude(c))
            s["out"] = [torch.empty(s[n].shape, dtype=s[n].dtype, device="cuda") for n in ("q", "k")]
            if c["mode"] == "step":
                s["grads"] = [torch.empty(s[n].shape, dtype=s[n].dtype, device="cuda") for n in ("q", "k")]
    s["case"] = c
    return s


# ---------------------------------------------------------------------------
# AdamW, plain: in 32 bits, the states' arithmetic operation by operation
# ---------------------------------------------------------------------------
def _hash(first, t):
    """32 random bits for every element of blocks, from its place in its tensor and the step."""
    x = (first[:, None] + torch.arange(BLOCK, device="cuda")) * 0x9E3779B1 + t * 0x6A09E667
    x &= 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    x = ((x ^ (x >> 13)) * 0x3C6EF373) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _scale_of(top, most):
    """(scale, its reciprocal) of blocks whose largest value is `top`: both 0 for blocks of
    values too small for 8 bits' reciprocal."""
    tiny = top < 2.0 ** -110
    return (torch.where(tiny, 0.0, top / torch.full_like(top, most)),
            torch.where(tiny, 0.0, torch.full_like(top, most) / top))


def _to_e4m3(m, r):
    """Codes and scales of signed values: rounded up where 16 random bits r say so."""
    scale, times = _scale_of(m.abs().amax(1), 448.0)
    x = m * times[:, None]
    a = x.abs()
    code = torch.where(a < 2.0 ** -6, ((a * 2.0 ** 25).int() + r) >> 16,
                       ((a.view(torch.int32) + (r << 4)) >> 20) - (120 << 3)).clamp_(max=0x7E)
    code |= (x < 0).int() << 7
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _to_e5m2(v, r):
    """The same for values that are not negative; a positive one does not become 0."""
    scale, times = _scale_of(v.amax(1), 57344.0)
    x = v * times[:, None]
    code = torch.where(x < 2.0 ** -14, ((x * 2.0 ** 32).int() + r) >> 16,
                       ((x.view(torch.int32) + (r << 5)) >> 21) - (112 << 2)).clamp_(max=0x7B)
    code = torch.where(x > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).view(torch.float8_e5m2), scale


def _adamw_group(s, t, clip):
    """One step, t the number of steps with it, clip the gradients' factor or None."""
    b1, b2 = BETAS
    step = LR / (1.0 - b1 ** t.double())
    root = torch.sqrt(1.0 - b2 ** t.double()).float()
    g = s["g"].float()
    if clip is not None:
        g = g * clip
    m, v = s["m"], s["v"]
    if s["bits"] == 8:
        m, v = m.float() * s["m_scale"][:, None], v.float() * s["v_scale"][:, None]
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * g * (1.0 - b2)
    w = s["master"] if s["master"] is not None else s["p"].float()
    w = w * (1.0 - LR * s["decay"]) - step.float() * m / (torch.sqrt(v) / root + EPS_ADAM)
    alone = s["master"] is None and s["p"].dtype == torch.bfloat16
    bits = _hash(s["first"], t) if alone or s["bits"] == 8 else None
    if alone:  # up or down in proportion
        rounded = (w.view(torch.int32) + (bits >> 16).int()) >> 16
        s["p"].copy_(rounded.to(torch.int16).view(torch.bfloat16))
    else:
        s["p"].copy_(w)
    if s["master"] is not None:
        s["master"].copy_(w)
    if s["bits"] == 8:
        (m, m_scale), (v, v_scale) = _to_e4m3(m, (bits & 0xFFFF).int()), _to_e5m2(v, (bits >> 16).int())
        s["m_scale"].copy_(m_scale)
        s["v_scale"].copy_(v_scale)
        s["m"].view(torch.uint8).copy_(m.view(torch.uint8))
        s["v"].view(torch.uint8).copy_(v.view(torch.uint8))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _adamw_outputs(s, norm):
    mats, vecs = s["groups"]
    got = {n: mats[n] for n in ("p", "master", "m", "v", "m_scale", "v_scale")}
    got.update(vec_p=vecs["p"], vec_m=vecs["m"], vec_v=vecs["v"], steps=s["steps"], norm=norm)
    return got


def _adamw_plain(s):
    mats, vecs = s["groups"]
    norm = clip = None
    if s["case"]["clip"]:
        norm = torch.sqrt(mats["g"].double().square().sum() + vecs["g"].double().square().sum())
        clip = (MAX_NORM / norm).clamp(max=1.0).float()
        norm = norm.float().reshape(1)
    s["steps"] += 1
    _adamw_group(mats, s["steps"], clip)
    _adamw_group(vecs, s["steps"], clip)
    return _adamw_outputs(s, norm)


# ---------------------------------------------------------------------------
# Layer norm, plain: in 32 bits, sums over rows in 64
# ---------------------------------------------------------------------------
def _norm_plain(s):
    dt = s["x"].dtype
    z = s["x"].float()
    if s["residual"] is not None:
        z = (z + s["residual"].float()).to(dt).float()
    mean = z.mean(-1, keepdim=True)
    d = z - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS_NORM)
    xh = d * rstd
    got = {"out": (xh * s["gamma"] + s["beta"]).to(dt), "mean": mean.squeeze(-1), "rstd": rstd.squeeze(-1)}
    if s["residual"] is not None:
        got["total"] = z.to(dt)
    if s["dy"] is None:
        return got
    dy = s["dy"].float()
    dxh = dy * s["gamma"]
    dz = (dxh - dxh.mean(-1, keepdim=True) - xh * (dxh * xh).mean(-1, keepdim=True)) * rstd
    if s["dtotal"] is not None:
        dz = dz + s["dtotal"].float()
    got.update(dx=dz.to(dt), dgamma=(dy * xh).sum((0, 1), dtype=torch.float64).float(),
               dbeta=dy.sum((0, 1), dtype=torch.float64).float())
    return got


# ---------------------------------------------------------------------------
# Rotary positions, plain: angles in 64 bits, the rest in 32
# ---------------------------------------------------------------------------
def _amplitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _frequencies(c):
    n, s = c["rot"] // 2, c["factor"]
    i = torch.arange(n, dtype=torch.float64, device="cuda")
    if c["scaling"] == "base":
        return (BASE * s ** (n / (n - 1))) ** (-i / n)
    f = BASE ** (-i / n)
    if c["scaling"] == "linear":
        return f / s
    if c["scaling"] == "parts":
        keep = ((ORIGINAL_LEN * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / s)
    return f


def _rotate(c, x, cos, sin):
    dt, r = x.dtype, c["rot"]
    x = x.float()
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1).to(dt)


def _rotary_plain(s):
    c = s["case"]
    pos = torch.arange(c["seq"], device="cuda")[None, :]
    if s["pos"] is not None:
        pos = pos + s["pos"][:, None]
    angle = pos.double()[:, :, None, None] * _frequencies(c)
    cos, sin = (torch.cos(angle) * _amplitude(c)).float(), (torch.sin(angle) * _amplitude(c)).float()
    got = {"q": _rotate(c, s["q"], cos, sin), "k": _rotate(c, s["k"], cos, sin)}
    if c["mode"] == "step":
        got.update(dq=_rotate(c, s["dq"], cos, -sin), dk=_rotate(c, s["dk"], cos, -sin))
    return got


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"adamw": _adamw_plain, "norm": _norm_plain, "rotary": _rotary_plain}[c["op"]](s)
    import paper_2202_11836_amd as P
    if c["op"] == "adamw":
        norm = s["optimizer"].step(LR, max_norm=MAX_NORM if c["clip"] else None)
        return _adamw_outputs(s, norm)
    if c["op"] == "norm":
        out, total, mean, rstd = P.layer_norm_forward(s["x"], s["gamma"], s["beta"], s["residual"],
                                                      eps=EPS_NORM, **s["out"])
        got = {"out": out, "mean": mean, "rstd": rstd}
        if c["residual"]:
            got["total"] = total
        if c["mode"] == "step":
            dx, dgamma, dbeta = P.layer_norm_backward(s["dy"], total, s["gamma"], mean, rstd,
                                                      dtotal=s["dtotal"], **s["grads"])
            got.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
        return got
    q, k = P.rotary_forward(s["rotary"], s["q"], s["k"], pos=s["pos"], q_out=s["out"][0], k_out=s["out"][1])
    got = {"q": q, "k": k}
    if c["mode"] == "step":
        got["dq"], got["dk"] = P.rotary_backward(s["rotary"], s["dq"], s["dk"], pos=s["pos"],
                                                 q_out=s["grads"][0], k_out=s["grads"][1])
    return got


# ---------------------------------------------------------------------------
# From the definitions in 64 bits
# ---------------------------------------------------------------------------
def _code64(x, mantissa, lowest, most, draw16):
    """x >= 0 as a float of `mantissa` bits and least exponent `lowest`, up where a draw of
    16 bits (0 .. 65535) and the part beyond the last bit come to one step or more."""
    _, e = torch.frexp(x)
    unit = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=lowest) - mantissa)
    part = torch.floor(x / unit + draw16 / 65536.0)
    return (part * unit).clamp(max=most)


def _draws64(sizes, step):
    """The 32 random bits of every element, block by block, by their definition."""
    def whole(t):
        return t & np.uint64(0xFFFFFFFF)

    place = np.concatenate([np.arange(-(-n // BLOCK) * BLOCK, dtype=np.uint64) for n in sizes])
    x = whole(place * np.uint64(0x9E3779B1) + np.uint64(step) * np.uint64(0x6A09E667))
    for shift, times in ((15, 0xBB67AE85), (13, 0x3C6EF373)):
        x = whole((x ^ (x >> np.uint64(shift))) * np.uint64(times))
    x ^= x >> np.uint64(16)
    return torch.from_numpy(x.astype(np.int64).reshape(-1, BLOCK)).cuda()


def _exact_group(t, step, clip):
    live = t["live"]
    g = t["g"].double() * clip
    m, v = t["m"].double(), t["v"].double()
    if t["bits"] == 8:
        m, v = m * t["m_scale"].double()[:, None], v * t["v_scale"].double()[:, None]
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
    w = (t["master"] if t["master"] is not None else t["p"]).double()
    w = w - LR * t["decay"] * w - LR * (m / (1 - BETAS[0] ** step)) / \
        (torch.sqrt(v / (1 - BETAS[1] ** step)) + EPS_ADAM)
    got = {"p": w, "master": w if t["master"] is not None else None, "m": m, "v": v, "m_scale": None,
           "v_scale": None}
    if t["bits"] == 8:
        bits = _draws64(t["sizes"], step)
        for name, most, mantissa, lowest, draw16 in (("m", 448.0, 3, -6, bits & 0xFFFF),
                                                     ("v", 57344.0, 2, -14, bits >> 16)):
            scale = got[name].abs().amax(1, keepdim=True) / most
            x = got[name] / torch.where(scale > 0, scale, torch.ones_like(scale))
            code = _code64(x.abs(), mantissa, lowest, most, draw16.double()) * torch.sign(x)
            if name == "v":
                code = torch.where(x > 0, code.clamp(min=2.0 ** -16), code)
            got[name], got[name + "_scale"] = code, scale.squeeze(1)
    if live is not None:  # nothing lies between tensors
        got = {n: x if x is None or x.dim() == 1 else x * live for n, x in got.items()}
    return got


def _exact_adamw(c, seed):
    s = _adamw_inputs(c, seed)
    mats, vecs = s["groups"]
    step, norm, clip = 21 + seed % 1000, None, 1.0
    if c["clip"]:
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t["g"].double().flatten())
                                                     for t in s["groups"]])).reshape(1)
        clip = torch.minimum(MAX_NORM / norm, torch.ones_like(norm))
    got, vec = _exact_group(mats, step, clip), _exact_group(vecs, step, clip)
    if c["dtype"] == "bf16_alone":
        # either neighbour of the exact value, by the draw
        bits = (_draws64(mats["sizes"], step) >> 16).double()
        a = got["p"].abs()
        got["p"] = _code64(a, 7, -126, math.inf, bits) * torch.sign(got["p"])
    got.update(vec_p=vec["p"], vec_m=vec["m"], vec_v=vec["v"], steps=None, norm=norm)
    return got


def _exact_norm(c, seed):
    s = _norm_inputs(c, seed)
    x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
    got = {}
    if c["residual"]:
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
        got["total"] = x
    n = c["width"]
    mu = x.sum(-1) / n
    rstd = (((x - mu[..., None]) ** 2).sum(-1) / n + EPS_NORM).rsqrt()
    xh = (x - mu[..., None]) * rstd[..., None]
    got.update(out=gamma * xh + beta, mean=mu, rstd=rstd)
    if c["mode"] == "step":
        dy = s["dy"].double()
        dxh = dy * gamma
        dx = rstd[..., None] / n * (n * dxh - dxh.sum(-1, keepdim=True) - xh * (dxh * xh).sum(-1, keepdim=True))
        if c["residual"]:
            dx = dx + s["dtotal"].double()
        got.update(dx=dx, dgamma=torch.einsum("bsc,bsc->c", dy, xh), dbeta=dy.sum((0, 1)))
    return got


def _exact_rotary(c, seed):
    """Each pair as a complex number, times that of its angle."""
    s = _rotary_inputs(c, seed)
    n, factor = c["rot"] // 2, c["factor"]
    freq = []
    for i in range(n):
        base = BASE * math.pow(factor, n / (n - 1)) if c["scaling"] == "base" else BASE
        f = math.pow(base, -i / n)
        if c["scaling"] == "linear":
            f /= factor
        elif c["scaling"] == "parts":
            turns = ORIGINAL_LEN * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - LOW) / (HIGH - LOW)))
            f = keep * f + (1 - keep) * f / factor
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    start = torch.zeros(c["batch"], device="cuda") if s["pos"] is None else s["pos"]
    pos = start.double()[:, None] + torch.arange(c["seq"], device="cuda")
    turn = torch.polar(torch.full((), _amplitude(c), dtype=torch.float64, device="cuda").expand(
        c["batch"], c["seq"], n), pos[..., None] * freq)[:, :, None]

    def rotated(x, turn):
        x = x.double()
        half = c["layout"] == "half"
        z = x[..., :2 * n].unflatten(-1, (2, n) if half else (n, 2))
        z = z.transpose(-1, -2) if half else z
        y = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        y = y.transpose(-1, -2) if half else y
        return torch.cat([y.flatten(-2), x[..., 2 * n:]], -1)

    got = {"q": rotated(s["q"], turn), "k": rotated(s["k"], turn)}
    if c["mode"] == "step":
        got.update(dq=rotated(s["dq"], turn.conj()), dk=rotated(s["dk"], turn.conj()))
    return got


def exact(case, seed):
    return {"adamw": _exact_adamw, "norm": _exact_norm, "rotary": _exact_rotary}[case["op"]](case, seed)
