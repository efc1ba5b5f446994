"""A stage with a relative position bias as programs run it: its step captured into a graph
and replayed with other inputs, masks and tables, and two such stages at once."""
import pytest
import torch

from paper_2202_11836_amd import Stage

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(shape, seed, dtype="f32"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).cuda()


def stage(dtype):
    st = Stage(2, 128, 2, 128, dtype=dtype, seed=8)
    st.set_relpos(16, 40)
    return st


def mask_of(B, S, seed):
    m = torch.rand((B, S), generator=torch.Generator().manual_seed(seed)) < 0.7
    m[seed % B] = False  # (a sequence without a key)
    return m.to(torch.uint8).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("noalloc", [False, True])
def test_step_in_a_graph(dtype, noalloc):
    B, S = 3, 150
    st, ref = stage(dtype), stage(dtype)
    x, dy = rand((B, S, 128), 0, dtype), rand((B, S, 128), 1, dtype)
    m, y, dx = mask_of(B, S, 0), torch.empty_like(x), torch.empty_like(x)

    def step():
        st.forward(x, m, out=y)
        if noalloc:
            st.backward_noalloc(dy, dx)
        else:
            st.backward(dy, dx)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    for i in range(4):
        x.copy_(rand((B, S, 128), 10 + i, dtype))
        dy.copy_(rand((B, S, 128), 20 + i, dtype))
        m.copy_(mask_of(B, S, i))
        for t in (st, ref):
            t.relpos_table().copy_(rand((16, 2), 30 + i))
        g.replay()
        torch.cuda.synchronize()
        yr = ref.forward(x, m)
        dxr = ref.backward(dy)
        assert torch.equal(y, yr) and torch.equal(dx, dxr)
        assert torch.equal(st.relpos_grad(), ref.relpos_grad())
        assert all(torch.equal(st.grad(l, j), ref.grad(l, j)) for l in range(2) for j in range(12))
    del g
    st.close()
    ref.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_stages_at_once(dtype):
    B, S = 3, 200
    pair, streams = (stage(dtype), stage(dtype)), (torch.cuda.Stream(), torch.cuda.Stream())
    xs = [rand((B, S, 128), i, dtype) for i in range(2)]
    want = []
    for st, x in zip(pair, xs):
        st.relpos_table().copy_(rand((16, 2), 5))
        y = st.forward(x)
        want.append((y, st.backward(y), st.relpos_grad().clone()))
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for st, x, s in zip(pair, xs, streams):
            with torch.cuda.stream(s):
                y = st.forward(x)
                got.append((y, st.backward(y)))
        torch.cuda.synchronize()
        for (y, dx), w, st in zip(got, want, pair):
            assert torch.equal(y, w[0]) and torch.equal(dx, w[1]) and torch.equal(st.relpos_grad(), w[2])
    for st in pair:
        st.close()
