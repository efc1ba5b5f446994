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
