"""Rotary positions against float64 within bounds derived from the formulas (_ops_ref.py): every
number of pairs in both layouts, positions to the ends of their type, layouts in memory, in
place, gradients, graphs and streams."""
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import DT, frequencies, rand, rotate, within

pytestmark = pytest.mark.gpu
LAYOUTS = ("half", "interleaved")


def check(rot, q, k=None, pos=None, freqs=None, **kw):
    freqs = frequencies(rot.rot_dim) if freqs is None else freqs
    for backward, fn in ((False, P.rotary_forward), (True, P.rotary_backward)):
        got = fn(rot, q, k, pos=pos, **kw)
        for name, x, y in (("q", q, got[0]), ("k", k, got[1])):
            if x is None:
                assert y is None
                continue
            want, tol = rotate(x, freqs, rot.layout, pos, rot.amplitude, backward)
            within((name, backward), y, want, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rot_dim", range(2, 66, 2))
def test_parts_of_the_head(rot_dim, layout, dtype):
    """Every number of pairs; what is behind them goes through bit for bit."""
    q, k = rand((2, 37, 3, 64), rot_dim, dtype), rand((2, 37, 1, 64), rot_dim + 1, dtype)
    rot = P.Rotary(rot_dim, layout=layout)
    check(rot, q, k)
    y, z = P.rotary_forward(rot, q, k)
    assert torch.equal(y[..., rot_dim:], q[..., rot_dim:]) and torch.equal(z[..., rot_dim:], k[..., rot_dim:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 0), (5, 1, 16, 4), (1, 2, 12, 12), (3, 77, 12, 3), (2, 513, 1, 1),
                                   (70, 40, 5, 5), (2, 9000, 2, 1), (1, 3, 128, 8), (9, 1, 300, 0),
                                   (1, 1200, 16, 16)], ids=str)
def test_shapes(shape, dtype):
    """One token to work-groups of many, few heads to more than a work-group has threads for."""
    B, S, H, G = shape
    q, k = rand((B, S, H, 64), 1, dtype), rand((B, S, G, 64), 2, dtype) if G else None
    for layout in LAYOUTS:
        check(P.Rotary(layout=layout), q, k)
    check(P.Rotary(22), q, k)
    pos = torch.randint(0, 5000, (B,), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()
    check(P.Rotary(), q, k, pos=pos)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("scaling", [None, "linear", "base", "parts"])
def test_scaling(scaling, layout):
    kw = dict(scaling=scaling, factor=7.5, original_len=2048)
    for rot_dim in (2, 20, 64):
        rot = P.Rotary(rot_dim, 5e5, layout, amplitude=1.2, low=2.0, high=20.0, **kw)
        freqs = frequencies(rot_dim, 5e5, low=2.0, high=20.0, **kw)
        check(rot, rand((1, 600, 4, 64), 1), rand((1, 600, 2, 64), 2),
              torch.tensor([30000], dtype=torch.int32, device="cuda"), freqs)


def test_given_frequencies():
    freqs = [0.0, 3.0, 1e-9, -0.25, 100.0]
    check(P.Rotary(10, layout="interleaved", freqs=freqs, amplitude=0.5), rand((2, 50, 4, 64), 1, "bf16"),
          freqs=freqs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(dtype):
    """The ends of the type, a million, and below zero; with tokens that pass the end."""
    ends = [0, 1, -1, -5, 131071, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31]
    pos = torch.tensor(ends, dtype=torch.int32, device="cuda")
    q, k = rand((len(ends), 3, 4, 64), 1, dtype), rand((len(ends), 3, 2, 64), 2, dtype)
    check(P.Rotary(), q, k, pos)
    each = pos[:, None].repeat(1, 3)
    each[:, 1] = 77
    check(P.Rotary(32, layout="interleaved"), q, k, each)
    # (a position each, in any order of memory, one row for all sequences)
    row = torch.tensor([9, -3, 40000], dtype=torch.int32, device="cuda")
    check(P.Rotary(), q, k, row[None].expand(len(ends), 3))
    check(P.Rotary(), q, k, torch.stack([row] * len(ends), 1).t())
    # (every second of a longer list)
    check(P.Rotary(), q, k, pos.repeat_interleave(2)[::2])


@pytest.mark.parametrize("rot_dim", [64, 32, 20, 6])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_of_a_projection(dtype, layout, rot_dim):
    """q and k turned where they lie in one packed projection; its other values stay."""
    B, S, H, G = 3, 45, 6, 2
    packed = rand((B, S, H + 2 * G, 64), 1, dtype)
    q, k = packed[:, :, :H], packed[:, :, H:H + G]
    rot = P.Rotary(rot_dim, layout=layout, amplitude=0.75)
    want, rest = P.rotary_forward(rot, q, k), packed[:, :, H + G:].clone()
    assert want[0].is_contiguous()
    got = P.rotary_forward(rot, q, k, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(packed[:, :, H + G:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(dtype):
    """[batch, head, position] memory, heads shared by stride 0, rows with room between them."""
    B, S, H = 2, 19, 4
    q = rand((B, H, S, 64), 1, dtype).transpose(1, 2)
    k = rand((B, S, 1, 64), 2, dtype).expand(B, S, H, 64)
    big = torch.full((S, B, H, 96), 7.0, device="cuda").to(DT[dtype])
    out = big.transpose(0, 1)[..., 16:80]
    rot = P.Rotary(48)
    check(rot, q, k)
    y, _ = P.rotary_forward(rot, q, k, q_out=out)
    want, tol = rotate(q, frequencies(48), "half", None)
    within("q", y, want, tol)
    assert (big[..., :16] == 7.0).all() and (big[..., 80:] == 7.0).all()


@pytest.mark.parametrize("shape", [(0, 5, 4, 2), (3, 0, 4, 2)])
def test_nothing(shape):
    B, S, H, G = shape
    q, k = P.rotary_forward(P.Rotary(), torch.empty((B, S, H, 64), device="cuda"),
                            torch.empty((B, S, G, 64), device="cuda"))
    assert q.shape == (B, S, H, 64) and k.shape == (B, S, G, 64)


def test_not_finite():
    """NaN and infinities reach their own pair alone, and go through unturned where they are
    behind the pairs."""
    for layout in LAYOUTS:
        for rot_dim in (64, 32, 20):
            q = rand((1, 8, 2, 64), 1)
            rot = P.Rotary(rot_dim, layout=layout)
            want = P.rotary_forward(rot, q)[0]
            bad = q.clone()
            bad[0, 3, 1, 1], bad[0, 3, 1, 63] = float("nan"), float("inf")
            got = P.rotary_forward(rot, bad)[0]
            n = rot_dim // 2
            pairs = {1, n + 1 if layout == "half" else 0}
            if rot_dim == 64:
                pairs |= {63, 31 if layout == "half" else 62}
            else:
                assert got[0, 3, 1, 63] == float("inf")
            keep = [i for i in range(63) if i not in pairs]
            assert torch.equal(got[0, 3, 1, keep], want[0, 3, 1, keep])
            assert got[0, 3, 1, 1].isnan()
            got[0, 3, 1] = want[0, 3, 1]
            assert torch.equal(got, want)


def test_backward_is_the_gradient():
    """<y, dy> grows along dx by <dx, dx>: y is linear in x, so differences are exact."""
    for layout in LAYOUTS:
        rot = P.Rotary(40, layout=layout, amplitude=1.3)
        x, dy = rand((2, 9, 3, 64), 1), rand((2, 9, 3, 64), 2)
        dx = P.rotary_backward(rot, dy)[0].double()
        for i in range(4):
            d = rand((2, 9, 3, 64), 10 + i)
            up = (P.rotary_forward(rot, d)[0].double() * dy.double()).sum()
            # (2 n values, each off by 8 roundings of values of size 1.3 * 2)
            bound = 8 * 2.0 ** -24 * 1.3 * 2 * 2 * (d.double().abs() * dy.double().abs().max()).sum()
            assert abs(up - (d.double() * dx).sum()) < bound


def test_scores_depend_on_the_distance():
    """Through attention: positions moved together give the same result."""
    q, k, v = (rand((2, 40, 4, 64), i) for i in range(3))
    rot, outs = P.Rotary(), []
    for start in (0, 1000):
        pos = torch.full((2,), start, dtype=torch.int32, device="cuda")
        qr, kr = P.rotary_forward(rot, q, k, pos=pos)
        outs.append(P.attn_forward(qr, kr, v)[0])
    # scores are off by 8 roundings of |q||k| / 8, the softmax by twice that of |v|
    bound = 2 * 2 * 8 * 2.0 ** -24 * (q.norm(dim=-1).max() * k.norm(dim=-1).max() / 8) * v.abs().max() * 4
    assert (outs[0] - outs[1]).abs().max() < bound


def test_offsets_beyond_32_bits():
    """A cache of 2.2 billion values, its first and last sequences."""
    B, S = 33, (1 << 20) + 9
    cache = torch.zeros((B, S, 1, 64), dtype=torch.bfloat16, device="cuda")
    x = rand((1, S, 1, 64), 1, "bf16")
    cache[0], cache[-1] = x[0], x[0]
    rot = P.Rotary()
    want = P.rotary_forward(rot, x)[0]
    P.rotary_forward(rot, cache, q_out=cache)
    assert torch.equal(cache[0], want[0]) and torch.equal(cache[-1], want[0])


@pytest.mark.parametrize("shape", [(4, 1, 8, 2), (2, 300, 4, 4)], ids=str)
def test_graph_and_streams(shape):
    B, S, H, G = shape
    q, k, pos = rand((B, S, H, 64), 1, "bf16"), rand((B, S, G, 64), 2, "bf16"), torch.zeros(B, dtype=torch.int32, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rot = P.Rotary(32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.rotary_forward(rot, q, k, pos=pos, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        P.rotary_forward(rot, q, k, pos=pos, q_out=qo, k_out=ko)
    for i in range(1, 4):
        q.copy_(rand(tuple(q.shape), 10 + i))
        k.copy_(rand(tuple(k.shape), 20 + i))
        pos.fill_(1000 * i)
        g.replay()
        torch.cuda.synchronize()
        want = P.rotary_forward(rot, q, k, pos=pos)
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    results = []
    for st in [torch.cuda.Stream() for _ in range(3)]:
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            results.append(P.rotary_forward(rot, q, k, pos=pos))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in results for a, b in zip(r, want))
