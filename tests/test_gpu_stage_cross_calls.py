"""What a cross-attention pass of a stage refuses of its tensors before anything is
launched, and what it gives back of its context."""
import pytest
import torch

from paper_2202_11836_amd import PARAM_NAMES, Stage, StageError

pytestmark = pytest.mark.gpu


def half(dtype="f32"):
    return Stage(None, 128, 2, 256, dtype=dtype, first_unit=0, n_units=1, seed=3)


def rand(shape, seed, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()


def test_tensors_of_other_shapes_refused():
    st, x, mem = half(), rand((2, 9, 128), 1), rand((2, 5, 128), 2)
    for out in (x[:1].clone(), x.bfloat16(), torch.empty(2, 128, 9, device="cuda").transpose(1, 2),
                torch.empty_like(x, device="cpu")):
        with pytest.raises(AssertionError):
            st.forward_cross(x, mem, out=out)
    y = st.forward_cross(x, mem)
    for dy in (y[:1].clone(), y[:, :8].contiguous(), y.reshape(18, 128)):
        with pytest.raises(AssertionError):
            st.backward_cross(dy)
    for kw in (dict(out=y[:1].clone()), dict(out=y.bfloat16()), dict(out_memory=mem[:, :4].contiguous()),
               dict(out_memory=torch.empty_like(mem, device="cpu"))):
        with pytest.raises(AssertionError):
            st.backward_cross(y, **kw)
    dx, dmem = st.backward_cross(y)  # (the context is still there)
    torch.cuda.synchronize()
    assert dx.shape == x.shape and dmem.shape == mem.shape
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_tensor_for_both_gradients_refused(dtype):
    st, x, mem = half(dtype), rand((2, 9, 128), 1, dtype), rand((2, 9, 128), 2, dtype)
    y = st.forward_cross(x, mem)
    both = torch.empty_like(x)
    with pytest.raises(StageError) as e:
        st.backward_cross(y, out=both, out_memory=both)
    assert e.value.status == 1 and "same memory" in str(e.value)
    dx, dmem = st.backward_cross(y)
    torch.cuda.synchronize()
    assert not torch.equal(dx, dmem)
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_contexts_queries(dtype):
    """Q = x W_q^T + b_q alone is what a cross-attention context holds under QKV; an
    ordinary pass after it has all three again."""
    st, x, mem = half(dtype), rand((2, 9, 128), 1, dtype), rand((2, 5, 128), 2, dtype)
    st.set_param(0, PARAM_NAMES.index("b_qkv"), rand((384,), 4))
    w, b = (st.param(0, PARAM_NAMES.index(n)).double().cpu() for n in ("W_qkv", "b_qkv"))
    st.forward_cross(x, mem)
    q = st.saved(0, 1, 18)
    assert q.shape == (18, 128)
    xs = x.double().cpu().reshape(18, 128)
    want = xs @ w.T + b
    # 128 products and the bias in fp32, and the rounding to the stage's type
    t = torch.finfo(x.dtype).eps / 2
    bound = 130 * 2.0 ** -24 * (xs.abs() @ w.T.abs() + b.abs()) * (1 + t) + t * want.abs()
    assert bool(((q.double().cpu() - want[:, :128]).abs() <= bound[:, :128]).all())
    st.forward(x)
    q = st.saved(0, 1, 18)
    assert q.shape == (18, 384)
    assert bool(((q.double().cpu() - want).abs() <= bound).all())
    st.close()
