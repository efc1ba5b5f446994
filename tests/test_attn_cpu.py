"""The attention operators without a device: the ABI's symbols, the buckets, and
every refusal of a call (all checks come before any device call)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2202_11836_amd as P
from _attn_ref import bucket
from paper_2202_11836_amd import binding as Bn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(Bn.LIB_PATH), reason="library not built")


def test_symbols():
    src = open(os.path.join(ROOT, "include", "attn.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = set(re.findall(r"\b(attn_[a-z_]+)\s*\(", src))
    assert names == set(Bn.EXPORTED_ATTN)
    lib = ctypes.CDLL(Bn.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


@pytest.mark.parametrize("num,far,both", [(32, 128, True), (32, 128, False), (4, 5, True),
                                          (2, 3, False), (2, 2048, False), (5, 9, False),
                                          (64, 512, False), (64, 64, False), (256, 2048, True),
                                          (256, 129, False), (254, 2048, True)])
def test_buckets(num, far, both):
    r = P.RelPos(num, far, both)
    for d in range(-far - 3, far + 4):
        assert r.bucket(d) == bucket(d, num, far, both), d
    last = (num // 2 if both else num) - 1
    assert r.bucket(-2 ** 63) == last
    assert r.bucket(2 ** 62) == (num - 1 if both else 0)


def test_buckets_of_the_usual_bias():
    """By hand: 32 buckets both ways up to 128: 16 to a direction, 8 of them exact,
    borders at 8 * 16^(j / 8)."""
    r = P.RelPos()
    assert [r.bucket(-d) for d in (0, 1, 7, 8, 11, 12, 15, 16, 22, 23, 31, 32, 45, 46, 63, 64, 90,
                                   91, 10000)] == \
        [0, 1, 7, 8, 8, 9, 9, 10, 10, 11, 11, 12, 12, 13, 13, 14, 14, 15, 15]
    assert [r.bucket(d) for d in (1, 7, 8, 16, 128)] == [17, 23, 24, 26, 31]


@pytest.mark.parametrize("num,far,both", [(1, 128, False), (0, 128, False), (-4, 128, True),
                                          (33, 128, True), (2, 128, True), (32, 16, False),
                                          (32, 8, True), (32, 2049, True), (257, 1000, False),
                                          (32, 0, False), (2 ** 31 - 1, 5, False)])
def test_bucket_refusals(num, far, both):
    with pytest.raises(P.StageError) as e:
        P.RelPos(num, far, both)
    assert e.value.status == 1


def shape(**kw):
    d = dict(dtype=1, batch=2, seq_q=5, seq_k=7, heads=4, kv_heads=2, causal=0, scale=0.125)
    for n, S, H in (("q", 5, 4), ("k", 7, 2), ("v", 7, 2), ("out", 5, 4), ("dout", 5, 4),
                    ("dq", 5, 4), ("dk", 7, 2), ("dv", 7, 2)):
        d[n] = (S * H * 64, H * 64, 64)
    assert set(kw) <= set(d)
    d.update(kw)
    flat = [x for v in d.values() for x in (v if isinstance(v, tuple) else (v,))]
    return Bn._ATTN_SHAPE.pack(*flat)


# Addresses that are never read: every call below is refused.
PTR = {n: (i + 1) << 20 for i, n in enumerate(
    ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "dtable", "ws", "table"))}


def call(backward, s, rp=None, ws_bytes=1 << 20, **ptr):
    lib = P.load_library()
    p = dict(PTR, mask=None, q_pos=None)
    if rp is None:
        p["table"] = p["dtable"] = None
    p.update(ptr)
    head = [s, ctypes.byref(rp) if rp is not None else None,
            p["table"], p["q"], p["k"], p["v"], p["mask"], p["q_pos"], p["out"], p["lse"]]
    if backward:
        st = lib.attn_backward(*head, p["dout"], p["dq"], p["dk"], p["dv"], p["dtable"], p["ws"],
                               ws_bytes, None)
    else:
        st = lib.attn_forward(*head, p["ws"], ws_bytes, None)
    return st, lib.attn_last_error().decode()


SHAPE_REFUSALS = [
    dict(dtype=2), dict(dtype=-1), dict(batch=-1), dict(seq_q=-1), dict(seq_k=-1),
    dict(seq_q=1 << 29), dict(seq_k=1 << 29), dict(heads=0), dict(kv_heads=0), dict(heads=5),
    dict(kv_heads=-2), dict(causal=2), dict(causal=-1), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(batch=1 << 24),
    dict(batch=2 ** 31 - 1, heads=2 ** 31 - 2, kv_heads=1),
    dict(q=(-1280, 256, 64)), dict(k=(896, -128, 64)), dict(v=(896, 128, -64)),
    dict(q=(1280, 257, 64)), dict(k=(899, 128, 64)), dict(v=(896, 128, 60)),
    dict(q=(1 << 62, 256, 64)), dict(q=(1280, 1 << 23, 64)),
    dict(out=(1280, 256, 0)), dict(out=(1280, 64, 64)), dict(out=(64, 256, 64)),
    dict(out=(1280, 255, 64)),
]


@pytest.mark.parametrize("kw", SHAPE_REFUSALS, ids=str)
@pytest.mark.parametrize("backward", [0, 1])
def test_shape_refusals(kw, backward):
    if backward and "out" in kw:
        kw = {"dq": kw["out"]}
    st, msg = call(backward, shape(**kw))
    assert st == 1 and msg, (st, msg)


def test_gradient_strides_refused():
    for kw in (dict(dk=(896, 128, 0)), dict(dv=(0, 128, 64)), dict(dq=(1280, 256, 32)),
               dict(dout=(1280, 256, 4)), dict(dk=(896, 64, 64))):
        st, msg = call(1, shape(**kw))
        assert st == 1 and msg


@pytest.mark.parametrize("name", ["q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"])
def test_pointers_refused(name):
    for value in (None, PTR[name] + 2):
        assert call(1, shape(), **{name: value})[0] == 1, value
        if name in ("q", "k", "v", "out") or (name == "lse" and value):
            assert call(0, shape(), **{name: value})[0] == 1, value


def test_outputs_over_inputs_refused():
    for o in ("q", "k", "v"):
        assert call(0, shape(), out=PTR[o])[0] == 1
    for o, i in (("dq", "q"), ("dk", "out"), ("dv", "dout"), ("dk", "dv"), ("dq", "dk")):
        assert call(1, shape(), **{o: PTR[i]})[0] == 1, (o, i)


def test_table_and_buckets_refused():
    rp = P.RelPos(32, 128).c
    assert call(0, shape(), rp, table=None)[0] == 1
    assert call(0, shape(), None, table=PTR["table"])[0] == 1
    assert call(0, shape(), rp, table=PTR["table"] + 1)[0] == 1
    assert call(1, shape(), None, dtable=PTR["dtable"])[0] == 1
    for field, value in (("num_buckets", 34), ("max_distance", 4000), ("bidirectional", 2),
                         ("reach", 128), ("reach", 1 << 20), ("n_borders", 8), ("n_borders", 127)):
        bad = Bn._RelPos.from_buffer_copy(rp)
        setattr(bad, field, value)
        assert call(0, shape(), bad)[0] == 1, field
        assert P.load_library().attn_relpos_bucket(ctypes.byref(bad), 3) == -1
    bad = Bn._RelPos.from_buffer_copy(rp)
    bad.border[2] = 1 << 20
    assert call(0, shape(), bad)[0] == 1
    assert call(0, shape(), Bn._RelPos())[0] == 1


def test_workspace():
    lib, n = P.load_library(), ctypes.c_size_t(7)
    s, rp = shape(), P.RelPos(32, 128).c
    assert lib.attn_workspace(s, None, 1, ctypes.byref(n)) == 0
    need = n.value
    assert need >= 2 * 4 * 5 * 4
    assert call(1, s, ws_bytes=need - 1)[0] == 1
    assert call(1, s, ws=None)[0] == 1
    assert call(1, s, ws=PTR["ws"] + 8)[0] == 1
    assert lib.attn_workspace(s, ctypes.byref(rp), 1, ctypes.byref(n)) == 0
    assert n.value >= need + 2 * 4 * 32 * 4
    assert call(1, s, rp, ws_bytes=n.value - 1)[0] == 1
    assert lib.attn_workspace(s, None, 2, ctypes.byref(n)) == 1
    assert lib.attn_workspace(s, None, 0, None) == 1
    assert lib.attn_workspace(None, None, 0, ctypes.byref(n)) == 1
    assert call(0, None)[0] == 1


def test_binding_refuses_cpu_tensors_and_wrong_types():
    q = torch.zeros(1, 2, 2, 64)
    for a in ((q, q, q), (q.half(), q, q), (q[..., :32], q, q), (q[0], q, q)):
        with pytest.raises(P.StageError):
            P.attn_forward(*a)


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_spans_beyond_any_memory_refused(name):
    """Strides that pass one by one, over so many sequences that their product would not."""
    inner = (256, 64) if name in ("q", "out") else (128, 64)
    st, msg = call(0, shape(batch=5000, **{name: (1 << 51, *inner)}))
    assert st == 1 and "spans" in msg
    st, msg = call(1, shape(batch=5000, **{"dq" if name == "out" else name: (1 << 52, *inner)}))
    assert st == 1 and "spans" in msg


def test_module_of_the_binding():
    """What the marshalling module says before any tensor is looked at."""
    P.RelPos()
    with pytest.raises(P.StageError):
        import torch
        P.attn_forward(*(torch.zeros(1, 2, 1, 64),) * 3)  # (sets the module up, refuses the CPU)
    from paper_2202_11836_amd import _attn_call as m
    for fn, n in ((m.forward, 11), (m.backward, 16), (m.setup, 12)):
        with pytest.raises(TypeError):
            fn(*(None,) * (n - 1))
    with pytest.raises(ValueError):
        m.setup(*(0,) * 12)
    for q in (None, 3, "q"):
        with pytest.raises(AttributeError):
            P.attn_forward(q, q, q)


def test_copies_of_the_buckets():
    import copy
    import pickle

    rp = P.RelPos(16, 50, False)
    for other in (copy.copy(rp), copy.deepcopy(rp), pickle.loads(pickle.dumps(rp))):
        assert other.addr != rp.addr and other.bidirectional is False
        assert [other.bucket(d) for d in range(-80, 9)] == [rp.bucket(d) for d in range(-80, 9)]
