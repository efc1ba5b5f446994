"""Plain implementations, in 64 bits, of layer norm, rotary positions and AdamW, with bounds
on how far a kernel that rounds as it says may be from them.

U[t] is the largest relative error of rounding to t once: half a step.  EPS counts fp32
roundings."""
import math

import torch

EPS = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


def rand(shape, seed, dtype="f32", std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(DT.get(dtype, dtype))


def within(name, got, want, tol):
    """Every value within its bound; NaN and infinities where they belong."""
    got, tol = got.double(), torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(want)
    assert got.shape == want.shape, name
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), name
    off = (got - want).abs()[fine]
    bad = off > tol[fine]
    assert not bad.any(), (name, off[bad].max().item(), tol[fine][bad][off[bad].argmax()].item(),
                           int(bad.sum()))


# ---------------------------------------------------------------------------
# Layer norm.  A row's sums go through at most 32 additions in a thread and 10 across
# threads, so a mean of values is off by 42 EPS of the mean of their sizes; the products and
# the final formula add a few.
# ---------------------------------------------------------------------------
K_ROW = 64


def norm_forward(x, gamma, beta, residual, eps):
    """(out, total, mean, rstd, tolerances of the three computed ones)"""
    z = x.double()
    if residual is not None:
        z = (x.float() + residual.float()).to(x.dtype).double()  # (one addition, rounded once or twice)
    mean = z.mean(-1)
    var = ((z - mean[..., None]) ** 2).mean(-1)
    rstd = (var + eps).rsqrt()
    xh = (z - mean[..., None]) * rstd[..., None]
    g = torch.ones(x.shape[-1], device=x.device) if gamma is None else gamma
    b = torch.zeros(x.shape[-1], device=x.device) if beta is None else beta
    g, b = g.double(), b.double()
    out = g * xh + b
    top = z.abs().amax(-1)
    off_mean = K_ROW * EPS * top
    # d (var) <= 2 |z - mean| off_mean on average; its root takes half of the relative error
    rel = K_ROW * EPS + off_mean * rstd * 2 * (var.sqrt() * rstd)
    off_xh = rstd[..., None] * (off_mean[..., None] + 2 * EPS * top[..., None]) + xh.abs() * rel[..., None]
    tol = U[x.dtype] * out.abs() + (1 + U[x.dtype]) * (g.abs() * off_xh + 4 * EPS * (b.abs() + out.abs()))
    return out, z, mean, rstd, (tol, off_mean, rstd * rel)


def norm_backward(dy, z, gamma, mean, rstd, dtotal):
    """(dx, dgamma, dbeta, their tolerances) from the fp32 mean and rstd."""
    d, mu, rs = dy.double(), mean.double()[..., None], rstd.double()[..., None]
    g = (torch.ones(dy.shape[-1], device=dy.device) if gamma is None else gamma).double()
    xh = (z.double() - mu) * rs
    wide = xh.abs() + (z.double().abs() + mu.abs()) * rs  # what xh's roundings are relative to
    dg = d * g
    dx = rs * (dg - dg.mean(-1, keepdim=True) - xh * (dg * xh).mean(-1, keepdim=True))
    part = rs * (dg.abs() + dg.abs().mean(-1, keepdim=True) + wide * (dg.abs() * wide).mean(-1, keepdim=True))
    tol = K_ROW * EPS * part
    if dtotal is not None:
        dx = dx + dtotal.double()
        tol = tol + 2 * EPS * dtotal.double().abs()
    tol = tol + U[dy.dtype] * (dx.abs() + tol)

    def rows(t):
        return t.reshape(-1, t.shape[-1]).sum(0)

    # (a column: at most 64 rows in a thread, 8 across threads, 48 of the work-groups' sums)
    k = 128 * EPS
    return dx, rows(d * xh), rows(d), (tol, k * rows(d.abs() * wide), k * rows(d.abs()))


# ---------------------------------------------------------------------------
# Rotary positions.  A cosine or sine is off by 4 EPS (its reduced angle's rounding, the series,
# the amplitude), a result by two more roundings; a position's angle, in 64 bits, by 2^-52 of it.
# ---------------------------------------------------------------------------
def frequencies(rot_dim, base=10000.0, scaling=None, factor=1.0, original_len=0, low=1.0, high=32.0):
    n, got = rot_dim // 2, []
    for i in range(n):
        b = base * factor ** (n / (n - 1)) if scaling == "base" and n > 1 else base
        f = b ** (-i / n)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            keep = min(1.0, max(0.0, (original_len * f / (2 * math.pi) - low) / (high - low)))
            f *= keep + (1 - keep) / factor
        got.append(f)
    return got


def positions(x, pos):
    B, S = x.shape[:2]
    at = torch.arange(S, device=x.device)[None, :].expand(B, S).double()
    if pos is None:
        return at
    return pos.double() if pos.dim() == 2 else at + pos.double()[:, None]


def rotate(x, freqs, layout, pos, amplitude=1.0, backward=False):
    """(turned, tolerance)"""
    n = len(freqs)
    f = torch.tensor(freqs, dtype=torch.float64, device=x.device)
    p = positions(x, pos)[:, :, None, None]
    a = p * f * (-1.0 if backward else 1.0)
    c, s = amplitude * torch.cos(a), amplitude * torch.sin(a)
    v = x.double()
    i = torch.arange(n, device=x.device)
    i0, i1 = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    y, tol = v.clone(), torch.zeros_like(v)
    x0, x1 = v[..., i0], v[..., i1]
    y[..., i0], y[..., i1] = x0 * c - x1 * s, x0 * s + x1 * c
    off = abs(amplitude) * (x0.abs() + x1.abs()) * (6 * EPS + 2.0 ** -51 * a.abs())
    tol[..., i0] = off + U[x.dtype] * (y[..., i0].abs() + off)
    tol[..., i1] = off + U[x.dtype] * (y[..., i1].abs() + off)
    return y, tol


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
def random_bits(n, t):
    x = (torch.arange(n, device=DEV) * 0x9E3779B1 + t * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    x = ((x ^ (x >> 13)) * 0x3C6EF373) & 0xFFFFFFFF
    return x ^ (x >> 16)


def adamw64(w, g, m, v, t, lr, betas, eps, decay, clip=1.0):
    """(w, m, v) after step t in 64 bits."""
    w, g, m, v = (x.double() for x in (w, g, m, v))
    g = g * clip
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    v = torch.where(v > torch.finfo(torch.float32).max, math.inf, v)  # (v is held in fp32)
    up = lr * (m / (1 - betas[0] ** t)) / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return w - lr * decay * w - up, m, v, up


def states32(g, m, v, betas, clip=None):
    """m and v in fp32, each operation rounded by itself: what the kernel forms, bit for bit."""
    g = g.float()
    if clip is not None:
        g = g * clip
    return m * betas[0] + g * (1.0 - betas[0]), v * betas[1] + g * g * (1.0 - betas[1])


def _blocks(x):
    n = x.numel()
    pad = torch.zeros(-n % 256, dtype=x.dtype, device=x.device)
    return torch.cat([x.reshape(-1), pad]).view(-1, 256)


def encode(x, kind, r):
    """(codes, scales) of a flat fp32 tensor, r its 16 random bits."""
    n, b = x.numel(), _blocks(x)
    most, mant, low = (448.0, 3, 6) if kind == "e4m3" else (57344.0, 2, 14)
    top = b.abs().amax(1)
    tiny = top < 2.0 ** -110
    scale = torch.where(tiny, 0.0, top / torch.full_like(top, most))
    inv = torch.where(tiny, 0.0, torch.full_like(top, most) / top)
    y = (b * inv[:, None]).reshape(-1)[:n]
    a = y.abs()
    drop = 23 - mant
    normal = ((a.view(torch.int32).long() + (r << (drop - 16))) >> drop) - ((127 - low - 1) << mant)
    small = ((a.double() * 2.0 ** (low + mant + 16)).long() + r) >> 16
    lost = ~torch.isfinite(top)  # (a value that is not finite: its block is NaN)
    scale = torch.where(lost, math.nan, scale)
    a = torch.where(lost.repeat_interleave(256)[:n], 0.0, a)
    y = torch.where(lost.repeat_interleave(256)[:n], 0.0, y)
    normal, small = torch.where(a > 0, normal, 0), torch.where(a > 0, small, 0)
    code = torch.where(a < 2.0 ** -low, small, normal).clamp(max=0x7E if kind == "e4m3" else 0x7B)
    if kind == "e4m3":
        code |= torch.signbit(y).long() << 7
    else:
        code = torch.where(y > 0, code.clamp(min=1), code)
    return code.to(torch.uint8), scale


def decode(codes, scale):
    """Flat fp32 values of float8 codes."""
    n = codes.numel()
    return (_blocks(codes.reshape(-1).float()) * scale[:, None]).reshape(-1)[:n]
