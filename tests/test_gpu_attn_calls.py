"""The attention operators as programs call them: in captured graphs, on streams of
their own, several at once, over caches beyond 32-bit offsets, into parts of larger
tensors, and what the binding refuses."""
import pytest
import torch

import paper_2202_11836_amd as P
from _attn_ref import check, reference
from paper_2202_11836_amd import StageError

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(shape, seed, dtype="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


class Case:
    """A call with everything in it, its buffers, and fresh values for them."""

    def __init__(self, dtype, B, H, G, Sq, Sk, relpos=None, causal=False, mask=False, step=True):
        self.shape, self.step = (B, H, G, Sq, Sk), step
        self.q, self.do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
        self.k, self.v = rand((B, Sk, 2, G, 64), 3, dtype).unbind(2)
        self.rp = P.RelPos(*relpos) if relpos else None
        self.relpos = relpos
        self.table = rand((relpos[0], H), 4) if relpos else None
        self.pos = torch.zeros(B, dtype=torch.int32, device="cuda") if causal else None
        self.mask = torch.ones((B, Sk), dtype=torch.uint8, device="cuda") if mask else None
        self.causal = causal
        self.out, self.lse = torch.empty_like(self.q), torch.empty((B, H, Sq), device="cuda")
        self.dq = torch.empty_like(self.q)
        self.dk, self.dv = torch.empty((B, Sk, 2, G, 64), dtype=self.q.dtype, device="cuda").unbind(2)
        self.dt = torch.empty_like(self.table) if relpos else None

    def fill(self, seed):
        B, H, G, Sq, Sk = self.shape
        for i, t in enumerate((self.q, self.do, self.k, self.v, self.table)):
            if t is not None:
                t.copy_(rand(tuple(t.shape), 100 * seed + i))
        if self.pos is not None:
            self.pos.copy_(torch.randint(-3, max(Sk - Sq, 1) + 3, (B,),
                                         generator=torch.Generator().manual_seed(seed)))
        if self.mask is not None:
            self.mask.copy_(torch.rand((B, Sk), generator=torch.Generator().manual_seed(seed)) < 0.7)

    def kw(self):
        return dict(key_mask=self.mask, causal=self.causal, q_pos=self.pos, relpos=self.rp,
                    table=self.table)

    def call(self):
        P.attn_forward(self.q, self.k, self.v, out=self.out, lse=self.lse, **self.kw())
        if self.step:
            P.attn_backward(self.q, self.k, self.v, self.out, self.lse, self.do, dq=self.dq,
                            dk=self.dk, dv=self.dv, dtable=self.dt, **self.kw())

    def results(self):
        r = [self.out, self.lse]
        if self.step:
            r += [self.dq, self.dk, self.dv] + ([self.dt] if self.dt is not None else [])
        return [t.clone() for t in r]

    def eager(self):
        out, lse = P.attn_forward(self.q, self.k, self.v, **self.kw())
        r = [out, lse]
        if self.step:
            r += [t for t in P.attn_backward(self.q, self.k, self.v, out, lse, self.do, **self.kw())
                  if t is not None]
        return r


# (every kernel: tiles, few queries with and without splits, both dQ and dK / dV splits)
CASES = [("bf16", 2, 4, 2, 300, 200, (32, 128), False, True, True),
         ("bf16", 1, 4, 4, 2, 3000, (32, 128, False), True, False, False),
         ("bf16", 2, 8, 2, 1, 500, None, True, True, False),
         ("bf16", 1, 2, 1, 700, 300, (16, 50, False), True, False, True),
         ("bf16", 1, 2, 2, 20, 2600, None, False, True, True),
         ("f32", 1, 2, 1, 400, 90, (32, 128), False, True, True),
         ("f32", 1, 2, 2, 20, 900, None, False, False, True)]


@pytest.mark.parametrize("args", CASES, ids=str)
def test_graph(args):
    """Captured once, replayed on new inputs, masks and positions, with eager work and
    other allocations in between."""
    c = Case(*args[:6], relpos=args[6], causal=args[7], mask=args[8], step=args[9])
    c.fill(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call()
    for i in range(1, 5):
        c.fill(i)
        g.replay()
        torch.cuda.synchronize()
        got, junk = c.results(), torch.full((1 << 22,), float("nan"), device="cuda")
        want = c.eager()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        del junk


def test_two_graphs_and_two_streams_at_once():
    """Two captured calls with partial results, replayed on two streams at the same
    time, and two eager ones likewise: each has a workspace of its own."""
    cases = [Case("bf16", 1, 4, 2, 900, 260, relpos=(32, 128)), Case("bf16", 1, 2, 2, 20, 2600, mask=True),
             Case("bf16", 1, 4, 4, 1, 4000, step=False)]
    want, streams, graphs = [], [torch.cuda.Stream() for _ in cases], []
    for i, c in enumerate(cases):
        c.fill(7 + i)
        want.append(c.eager())
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.call()
        graphs.append(g)
    for kind in ("graph", "eager"):
        for _ in range(5):
            for c in cases:
                for t in (c.out, c.dq):
                    t.zero_()
            torch.cuda.synchronize()
            for c, s, g in zip(cases, streams, graphs):
                with torch.cuda.stream(s):
                    g.replay() if kind == "graph" else c.call()
            torch.cuda.synchronize()
            for c, w in zip(cases, want):
                assert all(torch.equal(a, b) for a, b in zip(c.results(), w)), kind


@pytest.mark.parametrize("step", [False, True])
def test_offsets_beyond_32_bits(step):
    """Keys and values 8 KB apart in a 5 GB tensor: those that count lie behind 4 GiB
    (and at the start).  The same keys side by side give the reference."""
    H, Sk, n = 32, 600_000, 700
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    kv = torch.empty((1, Sk, 2, H, 64), dtype=torch.bfloat16, device="cuda")
    kv.fill_(float("nan"))
    mask = torch.zeros((1, Sk), dtype=torch.uint8, device="cuda")
    where = torch.cat([torch.arange(100), torch.arange(Sk - n + 100, Sk)]).cuda()
    near = rand((1, n, 2, H, 64), 5, "bf16")
    kv[:, where] = near
    mask[:, where] = 1
    for Sq in (1, 40) if not step else (70,):
        q, do = rand((1, Sq, H, 64), 6, "bf16"), rand((1, Sq, H, 64), 7, "bf16")
        k, v = kv.unbind(2)
        out, lse = P.attn_forward(q, k, v, key_mask=mask)
        kn, vn = near.unbind(2)
        want = reference(q, kn, vn, dout=do if step else None)
        check("out", out, want["out"])
        check("lse", lse, want["lse"])
        if step:
            dkv = torch.empty_like(kv)
            dk, dv = dkv.unbind(2)
            dq, _, _, _ = P.attn_backward(q, k, v, out, lse, do, key_mask=mask, dk=dk, dv=dv)
            check("dq", dq, want["dq"])
            check("dk", dk[:, where], want["dk"])
            check("dv", dv[:, where], want["dv"])
            dkv[:, where] = 0
            assert not dkv.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Sq,Sk", [(1, 300), (70, 130), (3, 33)])
def test_only_the_outputs_are_written(dtype, Sq, Sk):
    """Outputs inside larger tensors: what lies around and between their rows stays."""
    B, H, G = 2, 4, 2
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    mask = torch.ones((B, Sk), dtype=torch.uint8, device="cuda")
    mask[1, Sk // 2:] = 0

    def inside(S, heads):
        big = torch.full((B + 1, S + 9, heads + 1, 128), 7.0, dtype=DT[dtype], device="cuda")
        return big, big[:B, 4:4 + S, :heads, 32:96]

    bigs, parts = zip(*(inside(S, h) for S, h in ((Sq, H), (Sq, H), (Sk, G), (Sk, G))))
    lse_big = torch.full((B * H * Sq + 64,), 7.0, device="cuda")
    lse = lse_big[32:32 + B * H * Sq].view(B, H, Sq)
    P.attn_forward(q, k, v, key_mask=mask, out=parts[0], lse=lse)
    P.attn_backward(q, k, v, parts[0], lse, do, key_mask=mask, dq=parts[1], dk=parts[2], dv=parts[3])
    want = reference(q, k, v, mask=mask, dout=do)
    for n, t in zip(("out", "dq", "dk", "dv"), parts):
        check(n, t, want[n])
    check("lse", lse, want["lse"])
    for big, part in zip(bigs, parts):
        part.fill_(7.0)
        assert bool((big == 7.0).all())
    lse.fill_(7.0)
    assert bool((lse_big == 7.0).all())


def test_unaligned_and_broadcast_queries():
    """Strides with gaps, a head dimension of stride 0 and a batch of one sequence."""
    base = rand((1, 50, 3, 72), 1, "bf16")[..., 8:]
    q = base.expand(2, 50, 3, 64)
    k = rand((2, 40, 1, 64), 2, "bf16").expand(2, 40, 3, 64)
    v = rand((2, 1, 3, 64), 3, "bf16").expand(2, 40, 3, 64)
    do = rand((2, 1, 1, 64), 4, "bf16").expand(2, 50, 3, 64)
    out, lse = P.attn_forward(q, k, v)
    got = dict(zip(("dq", "dk", "dv"), P.attn_backward(q, k, v, out, lse, do)), out=out, lse=lse)
    want = reference(q, k, v, dout=do)
    for n in want:
        check(n, got[n], want[n])


def test_infinite_and_nan_inputs_stay_in_their_rows():
    """A NaN query has a NaN row and no other; a bias of -inf hides its bucket."""
    q, k, v = rand((1, 40, 2, 64), 1, "bf16"), rand((1, 70, 2, 64), 2, "bf16"), rand((1, 70, 2, 64), 3,
                                                                                  "bf16")
    clean, _ = P.attn_forward(q, k, v)
    q2 = q.clone()
    q2[0, 5, 1] = float("nan")
    out, lse = P.attn_forward(q2, k, v)
    bad = torch.zeros((1, 40, 2), dtype=torch.bool, device="cuda")
    bad[0, 5, 1] = True
    assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
    assert torch.equal(out[~bad], clean[~bad]) and bool(torch.isnan(lse[0, 1, 5]))
    rp = P.RelPos(4, 5)
    table = torch.tensor([[0.0] * 2, [0.0] * 2, [0.0] * 2, [float("-inf")] * 2], device="cuda")
    out, lse = P.attn_forward(q, k, v, relpos=rp, table=table)
    want = reference(q, k, v, mask=None, causal=True)  # bucket 3: every key after the query
    check("out", out, want["out"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Sq,Sk,q_pos", [(1, 300, [180, 3]), (5, 400, [200, -2]), (40, 200, [66, 0]),
                                         (150, 420, [100, -30]), (300, 640, [70, 200])])
@pytest.mark.parametrize("relpos", [None, (32, 128, False)])
def test_keys_that_no_query_reaches_yet(dtype, Sq, Sk, q_pos, relpos):
    """A cache is longer than what is in it: with `causal`, whatever lies behind the
    last query's position reaches nothing."""
    B, H, G = 2, 4, 2
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    for b, p in enumerate(q_pos):
        k[b, max(p + Sq, 0):], v[b, max(p + Sq, 0):] = float("nan"), float("inf")
    rp = P.RelPos(*relpos) if relpos else None
    table = rand((relpos[0], H), 5) if relpos else None
    kw = dict(causal=True, q_pos=torch.tensor(q_pos, dtype=torch.int32).cuda(), table=table)
    out, lse = P.attn_forward(q, k, v, relpos=rp, **kw)
    got = dict(zip(("dq", "dk", "dv", "dtable"),
                   P.attn_backward(q, k, v, out, lse, do, relpos=rp, **kw)), out=out, lse=lse)
    want = reference(q, k, v, relpos=relpos, dout=do, **kw)
    for n in want:
        check(n, got[n], want[n])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("relpos", [None, (32, 128, True), (32, 128, False)])
def test_positions_at_the_end_of_their_type(causal, relpos):
    """Every key is far before a query at 2^31 - 1, and far behind one at -2^31."""
    q, k, v = rand((2, 70, 2, 64), 1), rand((2, 130, 2, 64), 2), rand((2, 130, 2, 64), 3)
    do = rand((2, 70, 2, 64), 4)
    rp = P.RelPos(*relpos) if relpos else None
    table = rand((32, 2), 5) if relpos else None
    got, want = [], []
    for pos in ((2**31 - 1, -2**31), (10**6, -10**6)):
        kw = dict(causal=causal, q_pos=torch.tensor(pos).to(torch.int32).cuda(), table=table)
        out, lse = P.attn_forward(q, k, v, relpos=rp, **kw)
        got.append([out, lse, *P.attn_backward(q, k, v, out, lse, do, relpos=rp, **kw)])
        want = reference(q, k, v, relpos=relpos, dout=do, **kw)
    for a, b in zip(*got):
        assert a is b is None or torch.equal(a, b)
    for n, t in zip(("out", "lse", "dq", "dk", "dv"), got[1]):
        check(n, t, want[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,Sq,Sk", [(1, 2, 1, 1, 700), (2, 4, 4, 150, 130), (1, 2, 2, 3, 3000)])
def test_optional_results(dtype, B, H, G, Sq, Sk):
    """lse and dtable may be left out; the others are the same, up to the rounding that
    goes with the way D is formed."""
    import ctypes

    from paper_2202_11836_amd import binding as Bd

    lib = Bd.load_library()
    q, do = rand((B, Sq, H, 64), 1, dtype), rand((B, Sq, H, 64), 2, dtype)
    k, v = rand((B, Sk, G, 64), 3, dtype), rand((B, Sk, G, 64), 4, dtype)
    rp, table = P.RelPos(16, 60), rand((16, H), 5)
    out, lse = P.attn_forward(q, k, v, relpos=rp, table=table)
    st = [x for t in (q, k, v, q, do, q, k, v) for x in t.stride()[:3]]
    shape = Bd._ATTN_SHAPE.pack(1 if dtype == "bf16" else 0, B, Sq, Sk, H, G, 0, 0.125, *st)
    grads = [torch.full_like(t, float("nan")) for t in (q, k, v)]
    out2 = torch.full_like(q, float("nan"))

    def ws(backward):
        n = ctypes.c_size_t()
        assert lib.attn_workspace(shape, rp.ref, backward, ctypes.byref(n)) == 0
        return torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda"), n.value

    w, n = ws(0)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.attn_forward(shape, rp.ref, table.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                            None, None, out2.data_ptr(), None, w.data_ptr(), n, stream) == 0
    assert torch.equal(out, out2)
    w, n = ws(1)
    assert lib.attn_backward(shape, rp.ref, table.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                             None, None, out.data_ptr(), lse.data_ptr(), do.data_ptr(),
                             *(g.data_ptr() for g in grads), None, w.data_ptr(), n, stream) == 0
    want = reference(q, k, v, relpos=(16, 60, True), table=table, dout=do)
    for name, g in zip(("dq", "dk", "dv"), grads):
        check(name, g, want[name])


def test_binding_refusals():
    q, k = rand((2, 5, 4, 64), 1), rand((2, 7, 2, 64), 2)
    v, m = k.clone(), torch.ones((2, 7), dtype=torch.uint8, device="cuda")
    rp, t = P.RelPos(8, 20), torch.zeros((8, 4), device="cuda")
    out, lse = P.attn_forward(q, k, v)

    def refused(*a, **kw):
        with pytest.raises(StageError) as e:
            P.attn_forward(*a, **kw)
        assert e.value.status == 1 and str(e.value)

    refused(q, k, v[:, :6])
    refused(q, k.bfloat16(), v.bfloat16())
    refused(q, k.cpu(), v.cpu())
    refused(q.double(), k.double(), v.double())
    refused(q[..., :32], k[..., :32], v[..., :32])
    refused(q, k[:1], v[:1])
    refused(q[:, :, :3], k, v)                                 # 3 heads over 2
    refused(q, k, v, key_mask=m[:, :6])
    refused(q, k, v, key_mask=m.bool())
    refused(q, k, v, key_mask=torch.ones((7, 2), dtype=torch.uint8, device="cuda").t())
    refused(q, k, v, q_pos=torch.zeros(2, device="cuda"))
    refused(q, k, v, relpos=rp)
    refused(q, k, v, table=t)
    refused(q, k, v, relpos=rp, table=t[:, :3])
    refused(q, k, v, scale=0.0)
    refused(q, k, v, scale=float("nan"))
    refused(q, k, v, out=torch.empty_like(q).bfloat16())
    refused(q, k, v, out=q)
    refused(q, k, v, lse=torch.empty((2, 5, 4), device="cuda"))
    refused(q.transpose(2, 3).contiguous().transpose(2, 3), k, v)
    refused(q, torch.empty((2, 7, 2, 65), device="cuda")[..., 1:], v)   # rows 260 bytes apart
    refused(q, k, v, out=torch.empty((1, 5, 4, 64), device="cuda").expand(2, -1, -1, -1))
    with pytest.raises(StageError):
        P.attn_backward(q, k, v, out, lse, q, dtable=t)
    with pytest.raises(StageError):
        P.attn_backward(q, k, v, out, lse, q, dk=torch.empty((1, 7, 2, 64), device="cuda").expand(2, 7, 2, 64))
    with pytest.raises(StageError):
        P.attn_backward(q, k, v, out, lse, q, dq=out)


def test_scales_beyond_fp32_refused():
    q = rand((1, 2, 1, 64), 1)
    for scale in (1e39, float("inf"), -0.5):
        with pytest.raises(StageError) as e:
            P.attn_forward(q, q, q, scale=scale)
        assert e.value.status == 1


def test_references_are_given_back():
    """Calls that pass and calls that are refused, anywhere in their checks, keep no
    reference to what they were given, and none to what they made."""
    import gc
    import sys

    q, k = rand((2, 5, 4, 64), 1, "bf16"), rand((2, 7, 2, 64), 2, "bf16")
    v, do = rand((2, 7, 2, 64), 3, "bf16"), rand((2, 5, 4, 64), 4, "bf16")
    m, pos = torch.ones((2, 7), dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.int32,
                                                                              device="cuda")
    rp, table = P.RelPos(8, 20), torch.zeros((8, 4), device="cuda")
    out, lse = P.attn_forward(q, k, v)
    grads = [torch.empty_like(t) for t in (q, k, v)] + [torch.empty_like(table)]
    kw = dict(key_mask=m, scale=0.2, causal=True, q_pos=pos, relpos=rp, table=table)
    things = [q, k, v, do, m, pos, rp, table, out, lse, *grads, None, torch.float32, torch.bfloat16,
              torch.uint8, torch.int32, StageError]

    def calls():
        P.attn_forward(q, k, v)
        P.attn_forward(q, k, v, out=out, lse=lse, **kw)
        P.attn_backward(q, k, v, out, lse, do)
        P.attn_backward(q, k, v, out, lse, do, dq=grads[0], dk=grads[1], dv=grads[2], dtable=grads[3],
                        **kw)
        bad = torch.zeros(3, device="cuda")
        for a, b in [((q, k, bad), {}), ((bad, k, v), {}), ((q, bad, v), {}), ((q, k, v), dict(out=bad)),
                     ((q, k, v), dict(lse=bad)), ((q, k, v), dict(key_mask=bad)),
                     ((q, k, v), dict(q_pos=bad)), ((q, k, v), dict(relpos=rp, table=bad)),
                     ((q, k, v), dict(scale=-1.0)), ((q, k, v), dict(out=q))]:
            with pytest.raises(StageError):
                P.attn_forward(*a, **b)
        for b in (dict(dq=bad), dict(dk=bad), dict(dv=bad), dict(relpos=rp, table=table, dtable=bad),
                  dict(dtable=bad), dict(dq=out)):
            with pytest.raises(StageError):
                P.attn_backward(q, k, v, out, lse, do, **b)
        with pytest.raises(AttributeError):
            P.attn_forward(q, 3, v)
        with pytest.raises(TypeError):
            P.attn_forward(q, k, v, scale="much")

    # (tracebacks of refused calls are cycles that hold tensors until they are collected)
    calls()
    gc.collect()
    torch.cuda.synchronize()
    held, before = torch.cuda.memory_allocated(), [sys.getrefcount(t) for t in things]
    for _ in range(50):
        calls()
    gc.collect()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == held
    # (None and the types are held all over the interpreter)
    for t, n in zip(things, before):
        assert abs(sys.getrefcount(t) - n) < 20, t


def test_threads():
    """Calls from several threads at once, each on a stream of its own."""
    import threading

    cases = [Case(*c) for c in (CASES[0], CASES[2], CASES[4], CASES[5])]
    for i, c in enumerate(cases):
        c.fill(i)
    want = [c.eager() for c in cases]
    torch.cuda.synchronize()
    got, errors = [None] * len(cases), []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for n in range(30):
                    cases[i].call()
                    if n % 7 == 0:  # (and refused ones between them, with their messages)
                        try:
                            P.attn_forward(cases[i].q, cases[i].k, cases[i].v, scale=-1.0)
                        except StageError as e:
                            assert "scale" in str(e)
                got[i] = cases[i].results()
                torch.cuda.current_stream().synchronize()
        except BaseException as e:
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for g, w in zip(got, want):
        assert len(g) == len(w) and all(torch.equal(x, y) for x, y in zip(g, w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Sq,Sk", [(0, 5, 5), (0, 300, 700), (2, 0, 5), (2, 5, 0), (0, 0, 0)])
@pytest.mark.parametrize("relpos", [None, (8, 20, True)])
def test_nothing_to_do(dtype, B, Sq, Sk, relpos):
    q, k = rand((B, Sq, 4, 64), 1, dtype), rand((B, Sk, 2, 64), 2, dtype)
    rp = P.RelPos(*relpos) if relpos else None
    table = rand((8, 4), 3) if relpos else None
    out, lse = P.attn_forward(q, k, k.clone(), relpos=rp, table=table)
    assert out.shape == q.shape and not out.any() and bool((lse == float("-inf")).all())
    dq, dk, dv, dt = P.attn_backward(q, k, k.clone(), out, lse, q.clone(), relpos=rp, table=table)
    assert not dq.any() and not dk.any() and not dv.any() and (dt is None or not dt.any())
