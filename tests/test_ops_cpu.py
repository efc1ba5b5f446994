"""Layer norm, rotary positions and AdamW without a device: the ABI's symbols, the
frequencies, the random bits, and every refusal of a call (all checks come before any
device call)."""
import copy
import ctypes
import math
import os
import pickle
import re

import numpy as np
import pytest
import torch

import paper_2202_11836_amd as P
from _ops_ref import frequencies
from paper_2202_11836_amd import binding as Bn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(Bn.LIB_PATH), reason="library not built")
i32, i64, f32, f64, vp = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_void_p


def test_symbols():
    names = set()
    for h, prefix in (("norm.h", "layer_norm"), ("rotary.h", "rotary"), ("adamw.h", "adamw")):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(%s_[a-z_]+)\s*\(" % prefix, src))
    assert names == set(Bn.EXPORTED_OPS)
    lib = ctypes.CDLL(Bn.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kw", [{}, dict(scaling="linear", factor=8.0), dict(scaling="base", factor=16.0),
                                dict(scaling="parts", factor=4.0, original_len=8192),
                                dict(scaling="parts", factor=32.0, original_len=300, low=1.0, high=4.0),
                                dict(base=5e5)], ids=str)
@pytest.mark.parametrize("rot_dim", [2, 4, 20, 64])
def test_frequencies(rot_dim, kw):
    r = P.Rotary(rot_dim, **kw)
    want = frequencies(rot_dim, **kw)
    assert r.c.rot_dim == rot_dim and r.c.interleaved == 0 and r.c.amplitude == 1.0
    for got, f in zip(r.c.turns, want):
        assert abs(got * 2 * math.pi - f) <= 4e-15 * f
    assert all(t == 0 for t in list(r.c.turns)[rot_dim // 2:])


def test_given_frequencies_and_copies():
    r = P.Rotary(6, layout="interleaved", freqs=np.array([1.0, -0.5, 0.0]), amplitude=1.25)
    for x in (r, copy.deepcopy(r), pickle.loads(pickle.dumps(r)), copy.copy(r)):
        assert x.c.interleaved == 1 and x.c.amplitude == 1.25 and x.layout == "interleaved"
        assert np.allclose(np.array(x.c.turns[:3]) * 2 * math.pi, [1.0, -0.5, 0.0], rtol=1e-15, atol=0)
    assert copy.copy(r).addr != r.addr


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=66), dict(rot_dim=7), dict(rot_dim=-2),
                                dict(base=0.0), dict(base=-1.0), dict(base=math.nan), dict(layout="pairs"),
                                dict(scaling="far"), dict(scaling="linear", factor=0.0),
                                dict(scaling="base", factor=-1.0), dict(scaling="linear", factor=math.inf),
                                dict(scaling="parts", factor=2.0),
                                dict(scaling="parts", factor=2.0, original_len=100, low=3.0, high=3.0),
                                dict(scaling="parts", factor=2.0, original_len=100, low=math.nan),
                                dict(amplitude=math.inf), dict(amplitude=math.nan), dict(amplitude=1e39),
                                dict(freqs=[1.0]), dict(rot_dim=4, freqs=[1.0, math.nan]),
                                dict(rot_dim=4, freqs=[1.0, 1.0], scaling="linear", factor=2.0),
                                dict(base=1e-300, rot_dim=64, scaling="linear", factor=1e-300)], ids=str)
def test_rotary_refusals(kw):
    with pytest.raises(P.StageError) as e:
        P.Rotary(**kw)
    assert e.value.status == 1


class RotaryShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("heads", i32), ("kv_heads", i32),
                ("pos_each", i32)] + [(n, i64 * 3) for n in ("q", "k", "q_out", "k_out")] + [("pos", i64 * 2)]


# Addresses that are never read: every call below is refused.
A = {n: (i + 1) << 24 for i, n in enumerate(("q", "k", "q_out", "k_out", "pos"))}


def rotary_call(ptr=(), freqs=None, **kw):
    s = RotaryShape(1, 2, 5, 4, 2, 0, (i64 * 3)(1280, 256, 64), (i64 * 3)(640, 128, 64),
                    (i64 * 3)(1280, 256, 64), (i64 * 3)(640, 128, 64), (i64 * 2)(1, 0))
    for n, v in kw.items():
        setattr(s, n, type(getattr(s, n))(*v) if isinstance(v, tuple) else v)
    p = dict(A, **dict(ptr))
    lib = P.load_library()
    f = P.Rotary().c if freqs is None else freqs
    out = set()
    for fn in (lib.rotary_forward, lib.rotary_backward):
        fn.restype = i32
        st = fn(ctypes.byref(s), ctypes.byref(f) if f else None, vp(p["q"]), vp(p["k"]), vp(p["pos"]),
                vp(p["q_out"]), vp(p["k_out"]), None)
        out.add((st, lib.rotary_last_error().decode()))
    assert len(out) == 1
    return out.pop()


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=2), "dtype"), (dict(batch=-1), "negative"), (dict(seq=-1), "negative"), (dict(seq=1 << 29), "2^29"),
    (dict(heads=0), "heads"), (dict(kv_heads=-1), "heads"), (dict(heads=65535, kv_heads=1), "heads"),
    (dict(pos_each=2), "pos_each"), (dict(ptr={"q": None}), "null q"), (dict(ptr={"k_out": None}), "null k"),
    (dict(ptr={"q": A["q"] + 8}), "aligned"), (dict(ptr={"k_out": A["k_out"] + 2}), "aligned"),
    (dict(ptr={"pos": A["pos"] + 1}), "pos"), (dict(q=(1280, 252, 64)), "16 bytes"), (dict(k=(640, -128, 64)), "negative"),
    (dict(q=(1 << 54, 256, 64)), "16 bytes"), (dict(q=(1 << 53, 256, 64), batch=3), "2^53"),
    (dict(q_out=(1280, 128, 64)), "itself"), (dict(q_out=(1280, 256, 32)), "itself"), (dict(k_out=(0, 128, 64)), "itself"),
    (dict(ptr={"q_out": A["q"]}, q_out=(1280, 64, 320)), "same strides"),
    (dict(ptr={"q_out": A["k"]}), "another"), (dict(ptr={"k_out": A["q"]}), "another"),
    (dict(ptr={"k_out": A["q_out"]}), "another"), (dict(ptr={"q_out": A["pos"]}), "pos"),
    (dict(pos=(-1, 0)), "pos"), (dict(pos_each=1, pos=(1, -2)), "pos"), (dict(freqs=False), "frequencies"),
    (dict(freqs=Bn._RotaryFreqs(7, 0, 1.0)), "rot_dim"), (dict(freqs=Bn._RotaryFreqs(8, 2, 1.0)), "interleaved"),
    (dict(freqs=Bn._RotaryFreqs(8, 0, math.nan)), "amplitude"),
    (dict(batch=1 << 24, seq=2, heads=60, q=(7680, 3840, 64), k=(256, 128, 64), q_out=(7680, 3840, 64),
          k_out=(256, 128, 64)), "too large"),
], ids=str)
def test_rotary_call_refusals(kw, word):
    st, msg = rotary_call(**kw)
    assert st == 1 and word in msg, msg


def test_rotary_nothing_to_do():
    assert rotary_call(batch=0, ptr={n: None for n in A})[0] == 0
    assert rotary_call(seq=0)[0] == 0


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
class NormShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("width", i32), ("eps", f32)] + \
        [(n, i64 * 2) for n in ("x", "residual", "total", "out", "dy", "dtotal", "dx")]


N = {n: (i + 1) << 24 for i, n in enumerate(("x", "residual", "gamma", "beta", "total", "out", "mean", "rstd", "dy",
                                             "dtotal", "dx", "dgamma", "dbeta", "ws"))}


def norm_call(backward, ptr=(), ws_bytes=1 << 30, **kw):
    s = NormShape(1, 2, 5, 24, 1e-5, *[(i64 * 2)(120, 24) for _ in range(7)])
    for n, v in kw.items():
        setattr(s, n, (i64 * 2)(*v) if isinstance(v, tuple) else v)
    p = {n: vp(v) for n, v in dict(N, **dict(ptr)).items()}
    lib = P.load_library()
    if backward:
        lib.layer_norm_backward.restype = i32
        st = lib.layer_norm_backward(ctypes.byref(s), p["dy"], p["total"], p["gamma"], p["mean"], p["rstd"],
                                     p["dtotal"], p["dx"], p["dgamma"], p["dbeta"], p["ws"],
                                     ctypes.c_size_t(ws_bytes), None)
    else:
        lib.layer_norm_forward.restype = i32
        st = lib.layer_norm_forward(ctypes.byref(s), p["x"], p["residual"], p["gamma"], p["beta"], p["total"],
                                    p["out"], p["mean"], p["rstd"], None)
    return st, lib.layer_norm_last_error().decode()


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("kw,word", [
    (dict(dtype=-1), "dtype"), (dict(batch=-1), "negative"), (dict(seq=-2), "negative"), (dict(width=0), "width"),
    (dict(width=16385), "width"), (dict(batch=1 << 15, seq=1 << 16), "too large"),
    (dict(width=16384, batch=1 << 11, seq=1 << 11), "too large"),
    (dict(width=64, batch=1 << 15, seq=1 << 14), "too large"),
    (dict(ptr={"gamma": N["gamma"] + 2}), "aligned"), (dict(ptr={"mean": N["mean"] + 1}), "aligned")], ids=str)
def test_norm_refusals(kw, word, backward):
    st, msg = norm_call(backward, **kw)
    assert st == 1 and word in msg, msg


@pytest.mark.parametrize("kw,word", [
    (dict(eps=-1e-5), "eps"), (dict(eps=math.nan), "eps"), (dict(eps=math.inf), "eps"),
    (dict(ptr={"residual": None}), "without a residual"), (dict(ptr={"x": None}), "null x"),
    (dict(ptr={"out": None}), "null out"), (dict(ptr={"x": N["x"] + 1}), "x is not aligned"),
    (dict(x=(-120, 24)), "negative"), (dict(x=(1 << 53, 24)), "2^53"), (dict(out=(120, 23)), "itself"),
    (dict(out=(119, 24)), "itself"), (dict(total=(0, 24)), "itself"), (dict(total=(24, 47)), "itself"),
    (dict(ptr={"total": N["out"]}), "same memory"), (dict(ptr={"rstd": N["mean"]}), "same memory"),
    (dict(ptr={"out": N["gamma"]}), "input"), (dict(ptr={"mean": N["x"]}), "input"),
    (dict(ptr={"rstd": N["out"]}), "input"), (dict(ptr={"total": N["beta"]}), "input"),
    (dict(ptr={"out": N["x"]}, out=(24, 48)), "same strides"),
    (dict(ptr={"total": N["residual"]}, total=(24, 48)), "same strides")], ids=str)
def test_norm_forward_refusals(kw, word):
    st, msg = norm_call(0, **kw)
    assert st == 1 and word in msg, msg


@pytest.mark.parametrize("kw,word", [
    (dict(ptr={"dy": None}), "null dy"), (dict(ptr={"total": None}), "null total"),
    (dict(ptr={"mean": None}), "null mean"), (dict(dx=(120, 0)), "itself"),
    (dict(ptr={"dgamma": N["gamma"]}), "input"), (dict(ptr={"dbeta": N["dy"]}), "input"),
    (dict(ptr={"dgamma": N["dx"]}), "input"), (dict(ptr={"dx": N["mean"]}), "input"),
    (dict(ptr={"dgamma": N["dbeta"]}), "same memory"), (dict(ptr={"dx": N["dy"]}, dx=(24, 48)), "same strides"),
    (dict(ptr={"dx": N["dtotal"]}, dtotal=(240, 48)), "same strides"),
    (dict(ptr={"dx": N["total"]}, total=(240, 48)), "same strides"),
    (dict(ptr={"ws": None}), "workspace"), (dict(ws_bytes=191), "workspace"),
    (dict(ptr={"ws": N["ws"] + 4}), "workspace")], ids=str)
def test_norm_backward_refusals(kw, word):
    st, msg = norm_call(1, **kw)
    assert st == 1 and word in msg, msg


def test_norm_nothing_to_do():
    assert norm_call(0, batch=0, ptr={n: None for n in N})[0] == 0
    assert norm_call(1, batch=0, ptr={n: None for n in N})[0] == 0
    assert norm_call(1, ptr={"dx": None, "dgamma": None, "dbeta": None, "ws": None})[0] == 0


def test_norm_workspace():
    lib, n = P.load_library(), ctypes.c_size_t(7)
    lib.layer_norm_workspace.restype = i32
    for shape in ((0, 5, 64), (1, 1, 1), (32, 512, 1024), (2, 2500, 16384)):
        s = NormShape(1, *shape, 0.0)
        assert lib.layer_norm_workspace(ctypes.byref(s), ctypes.byref(n)) == 0
        rows, w = shape[0] * shape[1], shape[2]
        assert n.value % (8 * w) == 0 and n.value // (8 * w) <= rows and (n.value > 0) == (rows > 0)
    assert lib.layer_norm_workspace(ctypes.byref(s), None) == 1
    assert lib.layer_norm_workspace(None, ctypes.byref(n)) == 1


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
def adamw_init(steps=1 << 12, n=None, **kw):
    """adamw_init over one tensor of 1000 elements (or several: lists in kw)."""
    base = dict(param=1 << 20, grad=2 << 20, m=3 << 20, v=4 << 20, m_scale=None, v_scale=None, master=None,
                numel=1000, dtype=0, grad_dtype=0, state_bits=32, weight_decay=0.1, lr_scale=1.0)
    count = max([len(v) for v in kw.values() if isinstance(v, list)] + [1])
    t = (Bn._AdamWTensor * count)()
    for i in range(count):
        d = {k: (v[i] if isinstance(v, list) else v) for k, v in dict(base, **kw).items()}
        t[i] = Bn._AdamWTensor(**d)
    out, lib = vp(1), P.load_library()
    st = lib.adamw_init(t, count if n is None else n, vp(steps), ctypes.byref(out))
    assert out.value is None
    return st, lib.adamw_last_error().decode()


EIGHT = dict(state_bits=8, m_scale=5 << 20, v_scale=6 << 20)


@pytest.mark.parametrize("kw,word", [
    (dict(n=-1), "negative"), (dict(steps=None), "steps"), (dict(steps=4), "steps"), (dict(numel=-1), "negative"),
    (dict(numel=1 << 40), "2^40"), (dict(dtype=2), "type"), (dict(grad_dtype=-1), "type"),
    (dict(state_bits=16), "state_bits"), (dict(weight_decay=math.nan), "finite"), (dict(lr_scale=math.inf), "finite"),
    (dict(param=None), "null"), (dict(grad=None), "null"), (dict(m=None), "null"), (dict(v=None), "null"),
    (dict(EIGHT, m_scale=None), "null"), (dict(EIGHT, v_scale=None), "null"), (dict(m_scale=5 << 20), "scales"),
    (dict(master=5 << 20), "master"), (dict(param=(1 << 20) + 2), "aligned"), (dict(grad=(2 << 20) + 1), "aligned"),
    (dict(m=(3 << 20) + 1), "aligned"), (dict(EIGHT, v_scale=(6 << 20) + 2), "aligned"),
    (dict(dtype=1, master=(5 << 20) + 2), "aligned"), (dict(m=(1 << 20) + 3996), "share"),
    (dict(v=(3 << 20)), "share"), (dict(grad=(1 << 20)), "gradient"), (dict(grad=(3 << 20) + 3996), "gradient"),
    (dict(grad=(3 << 20) - 3996), "gradient"), (dict(param=[1 << 20, 1 << 20], m=[3 << 20, 7 << 20], v=[4 << 20, 8 << 20]), "share"),
    (dict(param=[1 << 20, 9 << 20], m=[3 << 20, 7 << 20], v=[4 << 20, 8 << 20], grad=[7 << 20, 2 << 20]), "gradient"),
    (dict(steps=3 << 20), "share")], ids=str)
def test_adamw_init_refusals(kw, word):
    st, msg = adamw_init(**kw)
    assert st == 1 and word in msg, msg


def test_adamw_null():
    lib = P.load_library()
    lib.adamw_step.restype = i32
    assert lib.adamw_init(None, 1, vp(8), ctypes.byref(vp())) == 1
    assert lib.adamw_init(None, 0, vp(8), None) == 1
    assert lib.adamw_step(None, None, None) == 1
    lib.adamw_destroy(None)


def bits_of(i, t):
    """By the definition, in Python's whole numbers."""
    x = (i * 0x9E3779B1 + t * 0x6A09E667) % 2 ** 32
    x = (x ^ x >> 15) * 0xBB67AE85 % 2 ** 32
    x = (x ^ x >> 13) * 0x3C6EF373 % 2 ** 32
    return x ^ x >> 16


def test_random_bits_are_fair():
    """Over elements, and over the steps of one element: the means of both halves, their
    product's (independent), and that of neighbours, within 5 deviations."""
    def look(x):
        lo, hi = (x & 0xFFFF) / 65536.0 - 0.5, (x >> 16) / 65536.0 - 0.5
        n = len(x)
        sd = 1 / 12 ** 0.5
        for u in (lo, hi):
            assert abs(u.mean()) < 5 * sd / n ** 0.5
            assert abs((u * u).mean() - 1 / 12) < 5 * (1 / 180) ** 0.5 / n ** 0.5
            for d in (1, 2, 64, 256):
                assert abs((u[d:] * u[:-d]).mean()) < 5 / 12 / n ** 0.5
        assert abs((lo * hi).mean()) < 5 / 12 / n ** 0.5

    def bits(i, t):
        x = (i * 0x9E3779B1 + t * 0x6A09E667) & 0xFFFFFFFF
        x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
        x = ((x ^ (x >> 13)) * 0x3C6EF373) & 0xFFFFFFFF
        return x ^ (x >> 16)

    n = np.arange(1 << 18, dtype=np.uint64)
    assert [int(b) for b in bits(n[:50], np.uint64(7))] == [bits_of(i, 7) for i in range(50)]
    for t in (1, 2, 1000, 123457):
        look(bits(n, np.uint64(t)).astype(np.int64))
    for i in (0, 1, 255, 1 << 20):
        look(bits(np.uint64(i), n[1:]).astype(np.int64))


@pytest.mark.parametrize("kw", [dict(grads=[]), dict(weight_decay=[0.1, 0.2]), dict(state_bits=4),
                                dict(state_bits=[8, 8]), dict(lr_scale=[])], ids=str)
def test_adamw_python_refusals(kw):
    """(tensors of the CPU are refused too)"""
    p = torch.zeros(5)
    with pytest.raises(P.StageError) as e:
        P.AdamW([p], **dict(dict(grads=[p.clone()]), **kw))
    assert e.value.status == 1
    with pytest.raises(P.StageError) as e:
        P.AdamW([p], [p.clone()])
    assert "cuda" in str(e.value) or "on cpu" in str(e.value)


def test_what_is_no_tensor_with_memory():
    """The marshalling module says so of objects, sparse tensors and those without memory."""
    import torch
    for x in (None, 3, "x", [1.0]):
        with pytest.raises(TypeError, match="not a tensor"):
            P.layer_norm_forward(x)
    for x in (torch.zeros(2, 3).to_sparse(), torch.zeros(2, 3, device="meta"), torch.zeros(2, 3),
              torch.zeros((1,) * 9)):
        with pytest.raises(P.StageError):
            P.layer_norm_forward(x)
    from paper_2202_11836_amd import _ops_call as m
    for fn in (m.setup, m.norm_forward, m.norm_backward, m.rotary, m.adamw):
        with pytest.raises(TypeError, match="arguments"):
            fn()


def adamw_of_cpu_tensors(monkeypatch, params, grads, **kw):
    """An AdamW over tensors of the CPU, without a handle: what it holds, and the marshalling of its step."""
    monkeypatch.setattr(P.AdamW, "_fits", lambda *a: None)
    monkeypatch.setattr(P.AdamW, "_make", lambda *a: None)
    return P.AdamW(params, grads, **kw)


def test_adamw_holds_memory_not_objects(monkeypatch):
    """What a module's cast or a new .data takes from a tensor stays the optimizer's memory."""
    net = torch.nn.Linear(300, 70)
    params, grads = list(net.parameters()), [torch.randn_like(p) for p in net.parameters()]
    opt = adamw_of_cpu_tensors(monkeypatch, params, grads)
    every = params + grads + opt.state["exp_avg"] + opt.state["exp_avg_sq"] + [opt.state["steps"]]
    at, was = [t.data_ptr() for t in every], [t.detach().clone() for t in every]
    net.double()
    for t in every[2:]:
        t.data = torch.full_like(t, 7)
    junk = [torch.full_like(t, 9) for t in was for _ in range(20)]
    held = {t.data_ptr(): t for t in opt._held}
    for a, w in zip(at, was):
        assert a in held and torch.equal(held[a], w)
    assert all((j == 9).all() for j in junk)


@pytest.mark.skipif(torch.cuda.is_available(), reason="a handle that is none")
@pytest.mark.parametrize("name,i", [("params", 0), ("params", 1), ("grads", 1), ("exp_avg", 0), ("exp_avg_sq", 1),
                                    ("exp_avg_scale", 0), ("master", 1), ("steps", None)])
@pytest.mark.parametrize("how", ["data", "offset", "resized"])
def test_adamw_step_of_moved_tensors(name, i, how, monkeypatch):
    """Refused before the handle is looked at, and no longer once the memory is back."""
    params = [torch.randn(300).bfloat16(), torch.randn(40, 20).bfloat16()]
    opt = adamw_of_cpu_tensors(monkeypatch, params, [torch.randn_like(p) for p in params], state_bits=8)
    opt.device = torch.device("cuda", 0)
    block = ctypes.create_string_buffer(4096)
    opt.handle = ctypes.addressof(block)
    own = {"params": opt.params, "grads": opt.grads, "steps": [opt.state["steps"]]}
    t = own.get(name, opt.state.get(name))[i or 0]
    back = t.data
    if how == "data":
        t.data = t.data.clone()
    elif how == "offset":
        t.data = t.data.view(-1)[1:]
    else:
        t.untyped_storage().resize_(0)
    try:
        with pytest.raises(P.StageError) as e:
            opt.step(1e-3)
        assert e.value.status == 1 and (name if i is None else f"{name}[{i}]") + " has other memory" in str(e.value)
        if how != "resized":
            t.data = back
            with pytest.raises((RuntimeError, AssertionError)) as e:  # (no device here)
                opt.step(1e-3)
            assert not isinstance(e.value, P.StageError)
    finally:
        opt.handle = None


def test_adamw_of_a_stage_that_is_gone():
    """Neither a step nor new master copies read a closed stage's memory, or an earlier bias table's."""
    class Gone:
        handle, _tables = None, 1

    opt = Bn._StageAdamW.__new__(Bn._StageAdamW)
    opt.stage, opt._tables, opt.handle = Gone(), 1, None
    opt.params, opt.state = [torch.ones(4).bfloat16()], {"master": [torch.zeros(4)]}
    for handle, tables, word in ((None, 1, "closed"), (5, 2, "table")):
        Gone.handle, Gone._tables = handle, tables
        for call in (opt.reset_master, lambda: opt.step(1e-3)):
            with pytest.raises(P.StageError) as e:
                call()
            assert e.value.status == 2 and word in str(e.value)
    assert (opt.state["master"][0] == 0).all()
    Gone._tables = 1
    opt.reset_master()
    assert (opt.state["master"][0] == 1).all()


class AdamWArgs(ctypes.Structure):
    _fields_ = [("lr", f32), ("lr_ptr", vp), ("beta1", f64), ("beta2", f64), ("eps", f32), ("max_norm", f32), ("norm", vp)]


@pytest.mark.parametrize("kw,word", [(dict(eps=0.0), "eps"), (dict(eps=9e-31), "eps"), (dict(eps=-1e-8), "eps"),
                                     (dict(eps=math.inf), "eps"), (dict(eps=math.nan), "eps"),
                                     (dict(beta2=1.0), "betas"), (dict(beta1=math.nan), "betas"),
                                     (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=math.nan), "max_norm"),
                                     (dict(lr=math.inf), "lr"), (dict(lr_ptr=6), "lr_ptr"), (dict(norm=64), "norm")], ids=str)
def test_adamw_step_refusals(kw, word):
    """(before the handle is looked at)"""
    lib, handle = P.load_library(), ctypes.create_string_buffer(4096)
    lib.adamw_step.restype = i32
    a = AdamWArgs(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8), **kw))
    assert lib.adamw_step(handle, ctypes.byref(a), None) == 1
    msg = lib.adamw_last_error().decode()
    assert word in msg, msg


def test_adamw_is_not_copied(monkeypatch):
    """A copy would share the handle, which both would free."""
    freed, p = [], torch.ones(4)
    opt = adamw_of_cpu_tensors(monkeypatch, [p], [p.clone()])
    monkeypatch.setattr(P.AdamW, "close", lambda self: freed.append(self.handle))
    opt.handle = 1 << 20
    try:
        for how in (copy.copy, copy.deepcopy, pickle.dumps):
            with pytest.raises(TypeError, match="state"):
                how(opt)
        assert 1 << 20 not in freed
    finally:
        opt.handle = None
