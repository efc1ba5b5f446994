"""Layer norm against float64 within bounds derived from its formulas (_ops_ref.py): widths of
every kernel variant and odd ones, rows that lie apart, broadcast or in place, gradients
against differences, graphs and streams, and what is left alone."""
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import DT, norm_backward, norm_forward, rand, within

pytestmark = pytest.mark.gpu


def run(shape, dtype, seed=0, residual=False, dtotal=False, gamma=True, beta=True, eps=1e-12, offset=0.3):
    """Forward and backward, each against its reference."""
    x = (rand(shape, seed) + offset).to(DT[dtype])
    res = rand(shape, seed + 1, dtype) if residual else None
    w = shape[-1]
    ga = 1 + rand((w,), seed + 2, std=0.2) if gamma else None
    be = rand((w,), seed + 3, std=0.2) if beta else None
    dy, dt = rand(shape, seed + 4, dtype), rand(shape, seed + 5, dtype) if dtotal else None
    out, total, mean, rstd = P.layer_norm_forward(x, ga, be, res, eps=eps)
    want, z, mu, rs, tol = norm_forward(x, ga, be, res, eps)
    assert torch.equal(total.double(), z)
    within("out", out, want, tol[0])
    within("mean", mean, mu, tol[1])
    within("rstd", rstd, rs, tol[2])
    dx, dg, db = P.layer_norm_backward(dy, total, ga, mean, rstd, dtotal=dt)
    wx, wg, wb, tol = norm_backward(dy, total, ga, mean, rstd, dt)
    within("dx", dx, wx, tol[0])
    within("dgamma", dg, wg, tol[1])
    within("dbeta", db, wb, tol[2])


# (each variant's narrowest and widest row, one more and one less than a vector, odd ones)
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 120, 128, 129, 255, 256, 257, 511, 512, 513, 765, 1000, 1024,
          1025, 1537, 2048, 2049, 4095, 4096, 4097, 5120, 8191, 8192, 8193, 12345, 16383, 16384]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, dtype):
    run((2, 9, width), dtype, seed=width, residual=width % 2 == 0, dtotal=width % 3 == 0,
        eps=1e-5 if width < 3 else 1e-12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 3, 7, 8, 33, 600, 4111, 20000])
def test_rows(rows, dtype):
    """From one row to more than work-groups with several passes."""
    for width in (64, 200, 1024) if rows > 600 else (40, 200, 768, 3000):
        run((rows, width), dtype, seed=rows + width, residual=True, dtotal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(9, 258), (9, 383), (2600, 384), (3001, 385), (9, 640), (8191, 514), (8192, 514),
                                        (8203, 599), (20000, 640), (8200, 767), (8192, 768), (8193, 769)])
def test_rows_in_three_chunks(rows, width, dtype):
    run((rows, width), dtype, seed=width, residual=rows % 2 == 1, dtotal=width % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(700, 1024), (701, 1024), (900, 2048), (901, 2048), (901, 4095), (1300, 4096),
                                        (1301, 4096), (1301, 5123)])
def test_weights_gradients_by_columns_and_by_partial_rows(rows, width, dtype):
    run((rows, width), dtype, seed=rows, dtotal=True)


@pytest.mark.parametrize("gamma", [False, True])
@pytest.mark.parametrize("beta", [False, True])
def test_without_weights(gamma, beta):
    run((5, 11, 96), "bf16", gamma=gamma, beta=beta)


@pytest.mark.parametrize("shape", [(37,), (3, 4, 5, 64), (2, 1, 3, 2, 24)])
def test_dimensions(shape):
    run(shape, "f32")


def test_far_from_zero():
    """A mean 1000 times the spread: the variance comes from centred values."""
    run((4, 50, 512), "f32", offset=1000.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [96, 101, 1024, 3001])
def test_rows_apart(width, dtype):
    """Operands that are parts of larger tensors, whose other values stay as they are."""
    B, S, pad = 3, 5, 13
    big = {n: torch.full((B, 2, S, width + pad), 7.0, device="cuda").to(DT[dtype]) for n in
           ("x", "res", "out", "total", "dy", "dt", "dx")}
    v = {n: t[:, 1, :, 3:3 + width] for n, t in big.items()}
    for i, n in enumerate(("x", "res", "dy", "dt")):
        v[n].copy_(rand((B, S, width), i))
    ga, be = 1 + rand((width,), 8, std=0.2), rand((width,), 9)
    out, total, mean, rstd = P.layer_norm_forward(v["x"], ga, be, v["res"], out=v["out"], total=v["total"])
    dx, dg, db = P.layer_norm_backward(v["dy"], total, ga, mean, rstd, dtotal=v["dt"], dx=v["dx"])
    want, z, mu, rs, tol = norm_forward(v["x"], ga, be, v["res"], 1e-12)
    assert torch.equal(v["total"].double(), z) and out is v["out"] and dx is v["dx"]
    within("out", v["out"], want, tol[0])
    wx, wg, wb, tol = norm_backward(v["dy"], v["total"], ga, mean, rstd, v["dt"])
    within("dx", v["dx"], wx, tol[0])
    within("dgamma", dg, wg, tol[1])
    within("dbeta", db, wb, tol[2])
    for n, t in big.items():
        rest = torch.ones(t.shape, dtype=torch.bool, device="cuda")
        rest[:, 1, :, 3:3 + width] = False
        assert (t[rest] == 7.0).all(), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 1100])
@pytest.mark.parametrize("base", [0, 8, 56, 248, 504, 1016, 1536])
def test_row_ends(base, rows, dtype):
    """Each number of values behind a row's last whole eight, between NaN that no result shows."""
    for width in range(base + 1, base + 8):
        big = {n: torch.full((rows, width + 9), float("nan"), device="cuda").to(DT[dtype]) for n in
               ("x", "res", "dy", "dt", "out", "dx")}
        v = {n: t[:, 5:5 + width] for n, t in big.items()}
        for i, n in enumerate(("x", "res", "dy", "dt")):
            v[n].copy_(rand((rows, width), width + i))
        ga, be = 1 + rand((width,), 8, std=0.2), rand((width,), 9)
        # (eps of one: narrow rows' values may lie close together, and then so do their gradients' terms)
        out, total, mean, rstd = P.layer_norm_forward(v["x"], ga, be, v["res"], eps=1.0, out=v["out"])
        want, z, mu, rs, tol = norm_forward(v["x"], ga, be, v["res"], 1.0)
        assert torch.equal(total.double(), z)
        within("out", out, want, tol[0])
        dx, dg, db = P.layer_norm_backward(v["dy"], total, ga, mean, rstd, dtotal=v["dt"], dx=v["dx"])
        wx, wg, wb, tol = norm_backward(v["dy"], total, ga, mean, rstd, v["dt"])
        within("dx", dx, wx, tol[0])
        within("dgamma", dg, wg, tol[1])
        within("dbeta", db, wb, tol[2])
        for n, t in big.items():
            assert t[:, :5].isnan().all() and t[:, 5 + width:].isnan().all(), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_transposed_and_broadcast(dtype):
    """Sequences side by side in memory, a residual shared by the batch, gradients of one row."""
    B, S, w = 4, 6, 200
    x = rand((S, B, w), 1, dtype).transpose(0, 1)
    res, dy = rand((1, S, w), 2, dtype).expand(B, S, w), rand((1, 1, w), 3, dtype).expand(B, S, w)
    ga = 1 + rand((w,), 4, std=0.2)
    out, total, mean, rstd = P.layer_norm_forward(x, ga, None, res)
    want, z, _, _, tol = norm_forward(x, ga, None, res, 1e-12)
    assert torch.equal(total.double(), z)
    within("out", out, want, tol[0])
    dx, dg, db = P.layer_norm_backward(dy, total, ga, mean, rstd)
    wx, wg, wb, tol = norm_backward(dy, total, ga, mean, rstd, None)
    within("dx", dx, wx, tol[0])
    within("dgamma", dg, wg, tol[1])
    within("dbeta", db, wb, tol[2])


@pytest.mark.parametrize("width", [72, 1024, 2500, 9000])
def test_in_place(width):
    x, res, dy, dt = (rand((3, 7, width), i, "bf16") for i in range(4))
    ga, be = 1 + rand((width,), 5, std=0.2), rand((width,), 6)
    plain = P.layer_norm_forward(x, ga, be, res)
    for over, over_total in (("x", "res"), ("res", "x"), (None, "x"), ("x", None)):
        t = {"x": x.clone(), "res": res.clone(), None: None}
        got = P.layer_norm_forward(t["x"], ga, be, t["res"], out=t[over], total=t[over_total])
        assert all(torch.equal(a, b) for a, b in zip(got, plain)), over
    one = x.clone()
    assert torch.equal(P.layer_norm_forward(one, ga, be, out=one)[0], P.layer_norm_forward(x, ga, be)[0])
    total, mean, rstd = plain[1:]
    want = P.layer_norm_backward(dy, total, ga, mean, rstd, dtotal=dt)
    for over in ("dy", "total", "dt"):
        t = {"dy": dy.clone(), "total": total.clone(), "dt": dt.clone()}
        got = P.layer_norm_backward(t["dy"], t["total"], ga, mean, rstd, dtotal=t["dt"], dx=t[over])
        assert got[0] is t[over] and all(torch.equal(a, b) for a, b in zip(got, want)), over


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [37, 1500])
@pytest.mark.parametrize("width", [3, 13, 493, 999, 1531, 2501, 8199])
def test_odd_rows_in_place(width, rows, dtype):
    """A row's last values are read with some of those before them, which may be written by then."""
    x, res, dy, dt = (rand((rows, width), i, dtype) for i in range(4))
    ga, be = 1 + rand((width,), 5, std=0.2), rand((width,), 6)
    want = P.layer_norm_forward(x, ga, be, res, eps=1e-5)
    a, b = x.clone(), res.clone()
    got = P.layer_norm_forward(a, ga, be, b, eps=1e-5, out=a, total=b)
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    _, total, mean, rstd = want
    want = P.layer_norm_backward(dy, total, ga, mean, rstd, dtotal=dt)
    for over in ("dy", "total", "dt"):
        t = {"dy": dy.clone(), "total": total.clone(), "dt": dt.clone()}
        got = P.layer_norm_backward(t["dy"], t["total"], ga, mean, rstd, dtotal=t["dt"], dx=t[over])
        assert all(torch.equal(s, t) for s, t in zip(got, want)), over


@pytest.mark.parametrize("rows", [1, 5, 3000])
def test_left_out(rows):
    x, dy = rand((rows, 300), 1), rand((rows, 300), 2)
    ga = 1 + rand((300,), 3, std=0.2)
    _, _, mean, rstd = P.layer_norm_forward(x, ga)
    dx, dg, db = P.layer_norm_backward(dy, x, ga, mean, rstd)
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = P.layer_norm_backward(dy, x, ga, mean, rstd, dx=None if want[0] else False,
                                    dgamma=None if want[1] else False, dbeta=None if want[2] else False)
        for g, w, t in zip(got, want, (dx, dg, db)):
            assert torch.equal(g, t) if w else g is None


@pytest.mark.parametrize("shape", [(0, 64), (3, 0, 64), (0, 5, 64)])
def test_no_rows(shape):
    x, ga = torch.empty(shape, device="cuda"), torch.ones(64, device="cuda")
    out, total, mean, rstd = P.layer_norm_forward(x, ga, ga)
    assert out.shape == shape and mean.shape == shape[:-1]
    dx, dg, db = P.layer_norm_backward(x, total, ga, mean, rstd, dgamma=torch.full((64,), 3.0, device="cuda"))
    assert dx.shape == shape and (dg == 0).all() and (db == 0).all()


def test_not_finite():
    """A row with a NaN or an infinity is NaN; the others are as without it."""
    x, dy = rand((6, 130), 1), rand((6, 130), 2)
    ga = 1 + rand((130,), 3, std=0.2)
    want = P.layer_norm_forward(x, ga)
    bad = x.clone()
    bad[1, 129], bad[4, 0] = float("nan"), float("inf")
    out, total, mean, rstd = P.layer_norm_forward(bad, ga)
    keep = [0, 2, 3, 5]
    assert torch.equal(out[keep], want[0][keep]) and out[[1, 4]].isnan().all()
    dx = P.layer_norm_backward(dy, total, ga, mean, rstd)[0]
    assert torch.equal(dx[keep], P.layer_norm_backward(dy, x, ga, *want[2:])[0][keep])


def test_constant_rows():
    """No spread: rstd = 1 / sqrt(eps), out = beta."""
    x, be = torch.full((5, 96), 3.0, device="cuda"), rand((96,), 1)
    out, _, mean, rstd = P.layer_norm_forward(x, None, be, eps=1e-6)
    assert torch.equal(out, be.expand(5, 96)) and (mean == 3.0).all()
    within("rstd", rstd, torch.full((5,), 1e3, device="cuda").double(), 1e3 * 4 * 2.0 ** -24)


@pytest.mark.parametrize("width", [5, 24, 130])
def test_differences(width):
    """The gradients against differences of the float64 formula."""
    x, dy, res, dt = (rand((3, width), i) for i in range(4))
    ga, be = 1 + rand((width,), 5, std=0.2), rand((width,), 6)
    eps = 1e-5
    _, total, mean, rstd = P.layer_norm_forward(x, ga, be, res, eps=eps)
    dx, dg, db = P.layer_norm_backward(dy, total, ga, mean, rstd, dtotal=dt)

    def value(x, ga, be):
        z = x + res.double()
        d = z - z.mean(-1, keepdim=True)
        out = ga * d * ((d * d).mean(-1, keepdim=True) + eps).rsqrt() + be
        return (out * dy.double()).sum() + (z * dt.double()).sum()

    args, h = [x.double(), ga.double(), be.double()], 1e-6
    for i, got in enumerate((dx, dg, db)):
        # (third derivatives h^2 / 6, of order rstd^3, and 1e-16 / h of rounding; fp32 sums)
        size = got.double().abs().max().item() + 1.0
        for at in range(0, args[i].numel(), 3):
            step = torch.zeros_like(args[i]).view(-1)
            step[at] = h
            step = step.view(args[i].shape)
            up = value(*[a + step if j == i else a for j, a in enumerate(args)])
            down = value(*[a - step if j == i else a for j, a in enumerate(args)])
            assert abs((up - down).item() / (2 * h) - got.view(-1)[at].item()) < 2e-5 * size


def test_offsets_beyond_32_bits():
    """2.2 billion values: the first and last rows, in place."""
    rows, w = (1 << 21) + 77, 1024
    x = torch.zeros((rows, w), dtype=torch.bfloat16, device="cuda")
    for s in (slice(0, 3), slice(rows - 3, rows)):
        x[s] = rand((3, w), 3, "bf16")
    ga = 1 + rand((w,), 5, std=0.2)
    want = norm_forward(x[-3:].clone(), ga, None, None, 1e-5)
    out, total, mean, rstd = P.layer_norm_forward(x, ga, eps=1e-5)
    within("out", out[-3:], want[0], want[4][0])
    assert torch.equal(out[:3], out[-3:])
    dx = P.layer_norm_backward(out, total, ga, mean, rstd, dx=out, dgamma=False, dbeta=False)[0]
    assert torch.equal(dx[:3], dx[-3:]) and dx[-3:].isfinite().all()


@pytest.mark.parametrize("shape", [(3, 65, 1000), (40, 1024), (2, 5000, 256)])
def test_graph_and_streams(shape):
    """Captured once, replayed on new inputs with eager work between; then two at once on streams
    of their own; the same bits every time."""
    w = shape[-1]
    ts = [rand(shape, i, "bf16") for i in range(4)]
    ga, be = 1 + rand((w,), 5, std=0.2), rand((w,), 6)
    out, total, dx = (torch.empty_like(ts[0]) for _ in range(3))
    dg, db = torch.empty_like(ga), torch.empty_like(be)

    def call(**to):
        o, t, mean, rstd = P.layer_norm_forward(ts[0], ga, be, ts[1], out=to.get("out"), total=to.get("total"))
        return (o, t) + P.layer_norm_backward(ts[2], t, ga, mean, rstd, dtotal=ts[3], dx=to.get("dx"),
                                              dgamma=to.get("dgamma"), dbeta=to.get("dbeta"))

    to = dict(out=out, total=total, dx=dx, dgamma=dg, dbeta=db)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(**to)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(**to)
    for i in range(1, 4):
        for j, t in enumerate(ts):
            t.copy_(rand(shape, 10 * i + j))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in to.values()]
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    streams, results = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for st in streams:
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                results.append(call())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in results for a, b in zip(r, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(1301, 8193), (1301, 8200), (1400, 16384), (2053, 12345)])
def test_wide_rows_by_partial_rows(rows, width, dtype):
    """Rows of more than 8192 values, more of them than the sums by columns take."""
    run((rows, width), dtype, seed=rows, dtotal=True)
