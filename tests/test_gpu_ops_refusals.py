"""What the binding of layer norm, rotary positions and AdamW refuses, with nothing launched:
types, shapes, devices, strides, and calls on what is closed."""
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import rand

pytestmark = pytest.mark.gpu


def refused(word, fn, *a, **kw):
    with pytest.raises(P.StageError) as e:
        fn(*a, **kw)
    assert e.value.status == 1 and word in str(e.value), str(e.value)


def test_norm():
    x, ga = rand((4, 6, 32), 1), torch.ones(32, device="cuda")
    f, b = P.layer_norm_forward, P.layer_norm_backward
    refused("bfloat16 or float32", f, x.half(), ga)
    refused("on a GPU", f, x.cpu(), ga)
    refused("gamma", f, x, ga.bfloat16())
    refused("gamma", f, x, ga[:31])
    refused("gamma", f, x, torch.ones(64, device="cuda")[::2])
    refused("beta", f, x, ga, ga.cpu())
    refused("residual", f, x, ga, ga, x.bfloat16())
    refused("residual", f, x, ga, ga, x[:, :5])
    refused("total without", f, x, ga, total=torch.empty_like(x))
    refused("out", f, x, ga, out=torch.empty_like(x)[:2])
    refused("side by side", f, rand((4, 32, 6), 1).transpose(1, 2), ga)
    refused("itself", f, x, ga, out=rand((4, 1, 32), 2).expand(4, 6, 32))
    refused("mean", f, x, ga, mean=torch.empty((6, 4), device="cuda").t())
    refused("rstd", f, x, ga, rstd=torch.empty((4, 6), device="cuda").bfloat16())
    refused("eps", f, x, ga, eps=-1.0)
    refused("width", f, torch.empty((3, 16385), device="cuda"))
    refused("width", f, torch.empty((3, 0), device="cuda"))
    refused("evenly spaced", f, rand((3, 4, 5, 32), 1).transpose(0, 1))
    refused("GPU", f, torch.zeros((), device="cuda"))
    _, total, mean, rstd = f(x, ga)
    refused("total", b, x, x.bfloat16(), ga, mean, rstd)
    refused("mean", b, x, x, ga, mean[:3], rstd)
    refused("dtotal", b, x, x, ga, mean, rstd, dtotal=x[:1])
    refused("dgamma", b, x, x, ga, mean, rstd, dgamma=torch.empty(31, device="cuda"))
    refused("over an input", b, x, x, ga, mean, rstd, dgamma=ga)
    refused("same strides", b, x[:, ::2], x[:, ::2], ga, mean[:, ::2].contiguous(), rstd[:, ::2].contiguous(),
            dx=x.view(-1)[:4 * 3 * 32].view(4, 3, 32))
    for bad in (3, "x", None):
        with pytest.raises((AttributeError, TypeError)):
            f(bad, ga)


def test_rotary():
    rot, q, k = P.Rotary(), rand((2, 5, 4, 64), 1), rand((2, 5, 2, 64), 2)
    for f in (P.rotary_forward, P.rotary_backward):
        refused("64", f, rot, rand((2, 5, 4, 32), 1))
        refused("64", f, rot, q[0])
        refused("bfloat16 or float32", f, rot, q.half())
        refused("GPU", f, rot, q.cpu())
        refused("of q", f, rot, q, k.bfloat16())
        refused("of q", f, rot, q, k[:, :4])
        refused("k_out without", f, rot, q, k_out=k)
        refused("heads", f, rot, q, k[:, :, :0])
        refused("side by side", f, rot, rand((2, 5, 64, 4), 1).transpose(2, 3))
        refused("pos", f, rot, q, k, pos=torch.zeros(3, dtype=torch.int32, device="cuda"))
        refused("pos", f, rot, q, k, pos=torch.zeros(2, dtype=torch.int64, device="cuda"))
        refused("pos", f, rot, q, k, pos=torch.zeros((2, 4), dtype=torch.int32, device="cuda"))
        refused("pos", f, rot, q, k, pos=torch.zeros(2, dtype=torch.int32))
        refused("q_out", f, rot, q, k, q_out=torch.empty_like(q).bfloat16())
        refused("heads of q", f, rot, q, k, q_out=torch.empty_like(k))
        refused("another", f, rot, q, q.clone(), k_out=q)
        refused("itself", f, rot, q, k, q_out=q[:, :, :1].expand_as(q))
        refused("same strides", f, rot, q, k, q_out=q.view(5, 2, 4, 64).transpose(0, 1))
        refused("aligned", f, rot, rand((641 * 64 + 1,), 1)[1:2561].view(2, 5, 4, 64))
        refused("16 bytes", f, rot, rand((2, 5, 4, 66), 1)[..., :64])
    with pytest.raises(AttributeError):
        P.rotary_forward(None, q)


def test_adamw():
    p, g = rand((300,), 1), rand((300,), 2)
    refused("gradients", P.AdamW, [p], [])
    refused("grads[0]", P.AdamW, [p], [g[:299]])
    refused("grads[0]", P.AdamW, [p], [g.half()])
    refused("params[0]", P.AdamW, [rand((600,), 1)[::2]], [g])
    refused("grads[0]", P.AdamW, [p], [g.cpu()])
    refused("params[1]", P.AdamW, [p, p.cpu()], [g, g])
    refused("share", P.AdamW, [p, p], [g, g])
    refused("share", P.AdamW, [p[:200], p[100:]], [g[:200], g[100:]])
    refused("gradient", P.AdamW, [p], [p])
    refused("finite", P.AdamW, [p], [g], weight_decay=float("nan"))
    o = P.AdamW([p], [g])
    for kw, word in ((dict(lr=float("nan")), "lr"), (dict(lr=torch.zeros(2, device="cuda")), "lr"),
                     (dict(lr=torch.zeros(1)), "lr"), (dict(lr=1e-3, max_norm=0), "max_norm"),
                     (dict(lr=1e-3, max_norm=-1.0), "max_norm"), (dict(lr=1e-3, max_norm=float("inf")), "max_norm")):
        refused(word, o.step, **kw)
    for kw, word in ((dict(betas=(1.0, 0.9)), "betas"), (dict(betas=(0.9, -0.1)), "betas"), (dict(eps=0.0), "eps")):
        refused(word, P.AdamW([p], [g], **kw).step, 1e-3)
    assert o.state["steps"].item() == 0
    for name, bad in (("exp_avg", [None]), ("exp_avg", [g[:10]]), ("exp_avg_scale", [g]), ("master", [g.clone()]),
                      ("exp_avg_sq", []), ("exp_avg_sq", [g.to(torch.float8_e5m2)])):
        refused(name, P.AdamW, [p], [g], state=dict(o.state, **{name: bad}))
    refused("steps", P.AdamW, [p], [g], state=dict(o.state, steps=torch.zeros(1, device="cuda")))
    o.close()
    o.close()
    refused("closed", o.step, 1e-3)
