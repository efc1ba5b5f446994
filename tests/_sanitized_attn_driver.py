"""Runs the attention operators' host code under AddressSanitizer and
UndefinedBehaviorSanitizer (launched by test_sanitized_attn.py with the sanitizer runtime
preloaded; argv[1] = the sanitized library): the buckets of every valid shape of bias
against their definition in whole numbers, workspace sizes over a wide range of shapes and
types, and refusals of both calls.  No device is touched and torch is not imported."""
import ctypes
import random
import struct
import sys

lib = ctypes.CDLL(sys.argv[1])
vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t


class RelPos(ctypes.Structure):  # attn_relpos
    _fields_ = [("num_buckets", i32), ("max_distance", i32), ("bidirectional", i32), ("reach", i32),
                ("n_borders", i32), ("border", i32 * 128)]


rp_p = ctypes.POINTER(RelPos)
lib.attn_relpos_init.argtypes = [i32, i32, i32, rp_p]
lib.attn_relpos_bucket.argtypes = [rp_p, i64]
lib.attn_workspace.argtypes = [ctypes.c_char_p, rp_p, i32, ctypes.POINTER(sz)]
lib.attn_forward.argtypes = [ctypes.c_char_p, rp_p] + [vp] * 9 + [sz, vp]
lib.attn_backward.argtypes = [ctypes.c_char_p, rp_p] + [vp] * 14 + [sz, vp]
lib.attn_last_error.restype = ctypes.c_char_p
EINVAL = 1


def check(cond, what):
    if not cond:
        print("FAILED:", what, flush=True)
        sys.exit(1)


def borders(num, far, both):
    """Least distances of the buckets behind the first half of a direction's."""
    n = num // 2 if both else num
    one = n // 2
    m, out, d = n - one, [], one
    for j in range(1, m):
        while d ** m < one ** (m - j) * far ** j:  # d / one < (far / one) ** (j / m)
            d += 1
        out.append(d)
    return one, out


def init(num, far, both):
    rp = RelPos()
    return lib.attn_relpos_init(num, far, both, ctypes.byref(rp)), rp


tried = 0
for both in (0, 1):
    for num in list(range(4 if both else 2, 40, 2)) + [64, 100, 254, 256] + ([] if both else [3, 5, 31, 255]):
        half = (num // 2 if both else num) // 2
        for far in sorted({half + 1, half + 2, 2 * half, 4 * half, 128, 512, 1000, 2047, 2048}):
            if not half < far <= 2048:
                continue
            st, rp = init(num, far, both)
            one, want = borders(num, far, both)
            check(st == 0 and list(rp.border[:rp.n_borders]) == want, (num, far, both))
            check(rp.reach == (want[-1] if want else one), ("reach", num, far, both))
            for d in (0, -1, 1, -one, one, -far, far, far + 1, -2 ** 63, 2 ** 63 - 1):
                b = lib.attn_relpos_bucket(ctypes.byref(rp), d)
                check(0 <= b < num, ("bucket", num, far, both, d))
            tried += 1
check(tried > 250, "buckets")
big = 2 ** 31 - 1
for args in ((1, 9, 0), (257, 999, 0), (33, 128, 1), (32, 16, 0), (32, 2049, 1), (32, 128, 2), (big, big, 0),
             (-big, -big, 1), (-2 ** 31, -2 ** 31, -2 ** 31)):
    check(init(*args)[0] == EINVAL, args)
check(lib.attn_relpos_init(32, 128, 1, None) == EINVAL, "null")

rng = random.Random(7)
SIZES = (0, 1, 2, 31, 64, 127, 129, 1000, 65537, 2 ** 20, 2 ** 29 - 1, 2 ** 29, big, -1)
rp = init(32, 128, 1)[1]


def pack(dtype, B, Sq, Sk, H, G, causal=0, scale=0.125, strides=None):
    return struct.pack("@7if24q", dtype, B, Sq, Sk, H, G, causal, scale,
                       *(strides or [rng.choice((0, 64, 128, 2 ** 40)) for _ in range(24)]))


ok = 0
for _ in range(20000):
    G = rng.choice((1, 2, 3, 8, 16, 128, 2 ** 20))
    s = pack(rng.choice((0, 1, 1, 0, 2)), rng.choice((0, 1, 3, 32, 1000, 2 ** 24, big)), rng.choice(SIZES),
             rng.choice(SIZES), min(big, G * rng.choice((1, 1, 2, 4, 1000))), G, rng.choice((0, 1)))
    n = sz(5)
    for backward in (0, 1):
        st = lib.attn_workspace(s, rng.choice((None, ctypes.byref(rp))), backward, ctypes.byref(n))
        check(st in (0, EINVAL) and n.value < 2 ** 62, "workspace")
        ok += st == 0
check(ok > 2000, ("valid shapes", ok))

# Every call below is refused: its workspace is missing or its strides are wrong.
PTR = [(i + 1) << 20 for i in range(16)]
for _ in range(20000):
    B, Sq, Sk, G = rng.randint(1, 9), rng.randint(1, 300), rng.randint(1, 300), rng.choice((1, 2, 4))
    H = G * rng.choice((1, 2))
    st = []
    for S, h in ((Sq, H), (Sk, G), (Sk, G), (Sq, H), (Sq, H), (Sq, H), (Sk, G), (Sk, G)):
        st += [S * h * 64, h * 64, 64]
    wrong = rng.randrange(12)  # (a stride of q, k, v or out)
    st[wrong] = rng.choice((-64, -2 ** 63, 3, 2 ** 54, 2 ** 63 - 8, 2 ** 62))
    s = pack(rng.choice((0, 1)), max(B, 2), max(Sq, 2), max(Sk, 2), max(2 * G, 2), 2 * G,
             rng.choice((0, 1)), strides=st)
    a = [None, PTR[0], PTR[1], PTR[2], None, None, PTR[3], PTR[4]]
    check(lib.attn_forward(s, None, *a, None, 0, None) == EINVAL, "forward")
    check(lib.attn_backward(s, None, *a, *PTR[5:9], None, None, 0, None) == EINVAL, "backward")
    check(lib.attn_last_error(), "message")
print("sanitized attention host paths: ok")
