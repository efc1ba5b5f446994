"""Runs the host code of layer norm, rotary positions and AdamW under AddressSanitizer and
UndefinedBehaviorSanitizer (launched by test_sanitized_ops.py with the sanitizer runtime
preloaded; argv[1] = the sanitized library): frequencies of every size and scaling, workspace
sizes, calls with nothing to do, and refusals over random arguments.  No device is touched and
torch is not imported."""
import ctypes
import math
import random
import sys

lib = ctypes.CDLL(sys.argv[1])
i32, i64, f32, f64, vp, sz = (ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_void_p,
                              ctypes.c_size_t)
EINVAL = 1


def check(cond, what):
    if not cond:
        print("FAILED:", what, flush=True)
        sys.exit(1)


class Freqs(ctypes.Structure):  # rotary_freqs
    _fields_ = [("rot_dim", i32), ("interleaved", i32), ("amplitude", f32), ("turns", f64 * 32)]


class RotaryShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("heads", i32), ("kv_heads", i32),
                ("pos_each", i32)] + [(n, i64 * 3) for n in ("q", "k", "q_out", "k_out")] + [("pos", i64 * 2)]


class NormShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("width", i32), ("eps", f32)] + \
        [(n, i64 * 2) for n in ("x", "residual", "total", "out", "dy", "dtotal", "dx")]


class AdamWTensor(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "master")] + \
               [("numel", i64), ("dtype", i32), ("grad_dtype", i32), ("state_bits", i32), ("decay", f32),
                ("lr_scale", f32)]


lib.rotary_init.argtypes = [i32, i32, f64, i32, f64, i32, f64, f64, f64, ctypes.POINTER(Freqs)]
lib.rotary_init_freqs.argtypes = [i32, i32, ctypes.POINTER(f64), f64, ctypes.POINTER(Freqs)]
lib.adamw_init.argtypes = [ctypes.POINTER(AdamWTensor), i32, vp, ctypes.POINTER(vp)]
rng = random.Random(3)

f = Freqs()
for dim in range(-2, 70):
    for scaling in range(-1, 5):
        for inter in (-1, 0, 1, 2):
            st = lib.rotary_init(dim, inter, 1e4, scaling, 4.0, 2048, 1.0, 32.0, 1.0, ctypes.byref(f))
            good = dim in range(2, 65, 2) and 0 <= scaling <= 3 and inter in (0, 1)
            check(st == (0 if good else EINVAL), ("rotary_init", dim, scaling, inter, st))
for base, factor, n, low, high, amp in ((math.nan, 1, 1, 1, 2, 1), (1e308, 1e308, 1, 1, 2, 1), (1e4, math.inf, 1, 1, 2, 1),
                                        (1e4, 2, 0, 1, 2, 1), (1e4, 2, 1, 2, 1, 1), (1e4, 2, 1, 1, 2, 1e300),
                                        (1e-320, 2, 1, 1, 2, 1)):
    for scaling in range(4):
        lib.rotary_init(64, 0, base, scaling, factor, n, low, high, amp, ctypes.byref(f))
check(lib.rotary_init(64, 0, 1e4, 0, 1, 1, 1, 2, 1, None) == EINVAL, "null out")
check(lib.rotary_init_freqs(64, 0, None, 1.0, ctypes.byref(f)) == EINVAL, "null freqs")
lib.rotary_init(64, 0, 1e4, 0, 1.0, 0, 0.0, 0.0, 1.0, ctypes.byref(f))

EDGE = [-2 ** 63, -1, 0, 1, 2, 3, 4, 7, 8, 64, 4096, 2 ** 29, 2 ** 31 - 1, 2 ** 53, 2 ** 62, 2 ** 63 - 1]
SMALL = [-2 ** 31, -1, 0, 1, 2, 3, 8, 1000, 65535, 65536, 2 ** 29, 2 ** 31 - 1]
calls = 0


def some(kind, n):
    return (i64 * n)(*[rng.choice(EDGE) for _ in range(n)])


# (a null pointer in every call that might otherwise be launched: refused, or nothing to do)
for _ in range(20000):
    s = RotaryShape(rng.choice((0, 1, 1, 2, -1)), rng.choice(SMALL), rng.choice(SMALL), rng.choice(SMALL),
                    rng.choice(SMALL), rng.choice((0, 1, 2)), some(i64, 3), some(i64, 3), some(i64, 3), some(i64, 3),
                    some(i64, 2))
    p = [rng.choice((None, 8, 16, 1 << 20)) for _ in range(5)]
    p[rng.choice((0, 3))] = None
    st = lib.rotary_forward(ctypes.byref(s), ctypes.byref(f), *map(vp, p), None)
    check(st == EINVAL or (st == 0 and 0 in (s.batch, s.seq)), ("rotary_forward", st))
    n = NormShape(rng.choice((0, 1, 2)), rng.choice(SMALL), rng.choice(SMALL), rng.choice(SMALL),
                  rng.choice((0.0, 1e-5, -1.0, math.nan)), *[some(i64, 2) for _ in range(7)])
    b = sz(0)
    st = lib.layer_norm_workspace(ctypes.byref(n), ctypes.byref(b))
    rows = n.batch * n.seq
    check(st in (0, EINVAL) and (st or b.value % 8 == 0) and (st or b.value <= 8 * 512 * n.width), "workspace")
    check(st or (b.value > 0) == (rows > 0), "workspace of no rows")
    p = [rng.choice((None, 2, 4, 1 << 20)) for _ in range(8)]
    p[rng.choice((0, 5))] = None
    st = lib.layer_norm_forward(ctypes.byref(n), *map(vp, p), None)
    check(st == EINVAL or (st == 0 and rows == 0), ("layer_norm_forward", st))
    p = [rng.choice((None, 2, 4, 1 << 20)) for _ in range(10)]
    p[rng.choice((0, 1))] = None
    if rows == 0:
        p[7] = p[8] = None  # (their zeros would be launched)
    st = lib.layer_norm_backward(ctypes.byref(n), *map(vp, p), sz(rng.choice((0, 64, 1 << 40))), None)
    check(st == EINVAL or (st == 0 and rows == 0), ("layer_norm_backward", st))
    calls += 4

for _ in range(3000):
    k = rng.randint(1, 5)
    t = (AdamWTensor * k)()
    for x in t:
        for name in ("param", "grad", "m", "v", "m_scale", "v_scale", "master"):
            setattr(x, name, rng.choice((None, rng.randrange(1, 1 << 40), rng.randrange(1, 1 << 36) * 16)))
        x.numel = rng.choice((0, 1, 255, 256, 100000, 2 ** 39, 2 ** 40, -1, 2 ** 63 - 1))
        x.dtype, x.grad_dtype, x.state_bits = rng.choice((0, 1)), rng.choice((0, 1)), rng.choice((8, 32))
        x.decay, x.lr_scale = rng.choice((0.0, 0.1)), 1.0
    t[rng.randrange(k)].state_bits = 7  # (one that is refused)
    out = vp(5)
    check(lib.adamw_init(t, k, vp(64), ctypes.byref(out)) == EINVAL and out.value is None, "adamw_init")
    # two of the same memory: all checks are gone through, and it is refused
    for x in t:
        x.state_bits = 32
        x.numel, x.dtype, x.grad_dtype, x.m_scale, x.v_scale, x.master = 100, 0, 0, None, None, None
        for j, name in enumerate(("param", "grad", "m", "v")):
            setattr(x, name, 4096 * (1 + j))
    check(lib.adamw_init(t, k, vp(64 if k > 1 else 4096), ctypes.byref(out)) == EINVAL, "adamw_init overlap")
    calls += 2
check(lib.adamw_step(None, None, None) == EINVAL, "adamw_step")
lib.adamw_destroy(None)
print("sanitized operators' host paths: ok,", calls, "calls")
