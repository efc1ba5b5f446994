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
