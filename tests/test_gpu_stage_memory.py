"""What a stage holds for passes that the attention operators make: nothing that grows
with the square of the sequence length."""
import pytest
import torch

from paper_2202_11836_amd import Stage

pytestmark = pytest.mark.gpu
H, F, S = 64, 64, 8192
SCORES = 4 * S * S  # bytes of one head's scores of one sequence


def x_of(S, dtype="f32", h=H, B=1):
    g = torch.Generator(device="cuda").manual_seed(3)
    return torch.randn(B, S, h, device="cuda", generator=g).to(
        torch.float32 if dtype == "f32" else torch.bfloat16)


def test_bias_holds_no_scores():
    st = Stage(2, H, 1, F, dtype="f32")
    st.set_relpos(32)
    y = st.forward(x_of(S))
    st.backward(y)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all()) and st.device_bytes() < SCORES
    st.close()


def test_cross_attention_holds_no_scores():
    st = Stage(None, H, 1, F, dtype="f32", first_unit=0, n_units=1)
    y = st.forward_cross(x_of(S), x_of(77))
    st.backward_cross(y)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all()) and st.device_bytes() < SCORES
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_passes_of_both_kinds_in_turn(dtype):
    """A pass of the stage's own attention after one that holds no scores (and no
    residual of the context) has its room again."""
    h, B = 128, 3
    half = dict(first_unit=0, n_units=1, dtype=dtype, seed=5)
    st, fresh = (Stage(None, h, 2, 256, **half) for _ in range(2))
    x, mem = x_of(70, dtype, h, B), x_of(33, dtype, h, B)
    want = fresh.forward(x)
    grad = fresh.backward(want)
    held = fresh.device_bytes()
    for _ in range(2):
        c = st.forward_cross(x, mem)
        st.backward_cross(c)
        y = st.forward(x)
        assert torch.equal(y, want) and torch.equal(st.backward(y), grad)
        st.set_relpos(8, 20)
        y = st.forward(x)
        st.backward(y)
        st.set_relpos(0)
    y = st.forward(x)
    assert torch.equal(y, want) and torch.equal(st.backward(y), grad)
    assert st.device_bytes() == held
    st.close()
    fresh.close()


def test_no_residual_of_the_context_with_a_bias():
    """bf16: less by that residual than without a bias, but for what the bias holds
    besides (table and gradient, the operators' workspace)."""
    L, h, B, S = 4, 512, 4, 128
    held = []
    for buckets in (0, 4):
        st = Stage(L, h, 8, 512, dtype="bf16")
        if buckets:
            st.set_relpos(buckets, 20)
        st.forward(x_of(S, "bf16", h, B))
        held.append(st.device_bytes())
        st.close()
    lo = L * B * S * h * 2
    # D, a row of bucket sums per work-group of 64 queries (keys in one piece), tables
    ws = 4 * (B * 8 * S + B * 8 * 2 * 4 + (L + 2) * 4 * 8) + 4096
    assert held[1] - held[0] <= ws - lo + 256 * L
