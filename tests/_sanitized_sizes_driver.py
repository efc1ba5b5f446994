"""Calls of layer norm and rotary positions with as many rows, tokens and sequences as their shapes hold,
under AddressSanitizer and UndefinedBehaviorSanitizer (launched by test_sanitized_sizes.py with the
sanitizer runtime preloaded; argv[1] = the sanitized library).  All are refused, or have nothing
to do: no device is touched, and torch is not imported."""
import ctypes
import sys

lib = ctypes.CDLL(sys.argv[1])
i32, i64, f32, f64, vp, sz = (ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_void_p,
                              ctypes.c_size_t)
TOP = 2 ** 31 - 1


class Freqs(ctypes.Structure):  # rotary_freqs
    _fields_ = [("rot_dim", i32), ("interleaved", i32), ("amplitude", f32), ("turns", f64 * 32)]


class RotaryShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("heads", i32), ("kv_heads", i32),
                ("pos_each", i32)] + [(n, i64 * 3) for n in ("q", "k", "q_out", "k_out")] + [("pos", i64 * 2)]


class NormShape(ctypes.Structure):
    _fields_ = [("dtype", i32), ("batch", i32), ("seq", i32), ("width", i32), ("eps", f32)] + \
        [(n, i64 * 2) for n in ("x", "residual", "total", "out", "dy", "dtotal", "dx")]


lib.rotary_init.argtypes = [i32, i32, f64, i32, f64, i32, f64, f64, f64, ctypes.POINTER(Freqs)]
lib.rotary_last_error.restype = lib.layer_norm_last_error.restype = ctypes.c_char_p
calls = 0


def refused(st, msg, word, what):
    global calls
    calls += 1
    if st != 1 or word not in msg.decode():
        print("FAILED:", what, st, msg, flush=True)
        sys.exit(1)


def at(*names):
    return [vp((i + 1) << 44) if n else None for i, n in enumerate(names)]


f = Freqs()
for rot_dim, inter in ((64, 0), (20, 0), (20, 1)):
    assert lib.rotary_init(rot_dim, inter, 1e4, 0, 1.0, 0, 0.0, 0.0, 1.0, ctypes.byref(f)) == 0
    for dtype in (0, 1):
        for batch, seq in ((TOP, 1), (TOP - 30, 1), (TOP - 1, 2), (TOP, 2 ** 29 - 1), (70000, 2 ** 29 - 1)):
            for heads, kv in ((1, 0), (9, 7), (65535, 0), (1, 65534)):
                q, k = (i64 * 3)(seq * heads * 64, heads * 64, 64), (i64 * 3)(seq * kv * 64, kv * 64, 64)
                if batch * seq * heads * 64 > 2 ** 53 or batch * seq * kv * 64 > 2 ** 53:
                    continue
                for pos, each in ((None, 0), (vp(1 << 50), 0), (vp(1 << 50), 1)):
                    s = RotaryShape(dtype, batch, seq, heads, kv, each, q, k, q, k, (i64 * 2)(seq, 1))
                    a = at(1, kv, 1, kv)
                    for fn in (lib.rotary_forward, lib.rotary_backward):
                        st = fn(ctypes.byref(s), ctypes.byref(f), a[0], a[1], pos, a[2], a[3], None)
                        refused(st, lib.rotary_last_error(), "too large", (batch, seq, heads, kv))

for dtype in (0, 1):
    for width in (1, 64, 300, 1000, 8192, 16384):
        for batch, seq in ((TOP, TOP), (TOP, 1), (1, TOP), (TOP, 2), (65536, 65536)):
            st2 = (i64 * 2)(seq * width, width)
            s = NormShape(dtype, batch, seq, width, 1e-5, st2, st2, st2, st2, st2, st2, st2)
            a, n = at(*[1] * 9), sz()
            refused(lib.layer_norm_forward(ctypes.byref(s), *a[:8], None), lib.layer_norm_last_error(), "too large", (batch, seq))
            refused(lib.layer_norm_backward(ctypes.byref(s), *a[:9], a[0], a[1], sz(1 << 40), None),
                    lib.layer_norm_last_error(), "too large", (batch, seq))
            refused(lib.layer_norm_workspace(ctypes.byref(s), ctypes.byref(n)), lib.layer_norm_last_error(), "too large", batch)
        most = 4294967040 // max(8, min(1024, width // 16))
        for rows in (most // 4, most // 2, 2 ** 22):  # (host arithmetic alone)
            s.batch, s.seq = 1, rows
            lib.layer_norm_workspace(ctypes.byref(s), ctypes.byref(n))
            calls += 1
print("sanitized sizes: ok,", calls, "calls")
