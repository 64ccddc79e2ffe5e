"""The host side of the output layers' and the beam search's calls, without a GPU: what they
refuse and say, what they launch on which stream, and what a failing call returns. The
library's objects are linked with the stand-in for the CUDA runtime."""
import ctypes
import os
import subprocess

import pytest

from paper_1904_03409_gb300 import binding, build

HERE = os.path.dirname(os.path.abspath(__file__))
USER, OTHER = 0x77, 0x99
OK, ARG, CUDA, UNSUPPORTED = 0, 1, 5, 7
FP32, BF16 = 0, 1
vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float


@pytest.fixture(scope="module")
def real():
    build.build()
    return binding.load()


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    build.build()
    so = str(tmp_path_factory.mktemp("fake") / "libstacklstm_fake.so")
    include = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include")
    objs = [os.path.join(build.BUILD, os.path.basename(s)[:-3] + ".o") for s in build.sources()]
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I" + include,
                           os.path.join(HERE, "fake_cudart.cpp"), *objs, "-lpthread", "-o", so])
    lib = ctypes.CDLL(so)
    lib.fake_calls.restype = lib.fake_unjoined.restype = ctypes.c_long
    lib.fake_fail_at.argtypes = [ctypes.c_long]
    lib.fake_log.restype = lib.stacklstm_op_last_error.restype = ctypes.c_char_p
    lib.stacklstm_op_last_error.argtypes = [vp]
    P = ctypes.POINTER(vp)
    for name, types in {"norm_create": [P, ci, ci, ci, ci, vp], "linear_create": [P] + [ci] * 6 + [vp],
                        "distill_create": [P] + [ci] * 5 + [vp], "beam_create": [P] + [ci] * 7 + [vp],
                        "norm_forward": [vp, ci, vp, vp, vp, cf, vp, vp, vp], "norm_backward": [vp, ci] + [vp] * 8,
                        "linear_forward": [vp, ci] + [vp] * 6, "linear_backward": [vp, ci] + [vp] * 8,
                        "distill_run": [vp, ci] + [vp] * 4 + [cf] * 3 + [vp] * 2, "beam_lse": [vp] * 3,
                        "beam_select": [vp] * 8, "beam_reorder": [vp] * 10, "beam_push": [vp] * 9,
                        "op_status": [vp], "op_destroy": [vp], "op_set_stream": [vp, vp]}.items():
        getattr(lib, "stacklstm_" + name).argtypes = types
    return lib


SIZES = {"norm": (40, 24), "linear": (40, 24, 16, 2), "distill": (40, 24, 3), "beam": (5, 8, 24, 7, 16)}


def create(lib, kind, dtype=BF16, sizes=None):
    h = vp()
    s = sizes or SIZES[kind]
    tail = (dtype, s[3], 0, USER) if kind == "linear" else (dtype, 0, USER)
    args = s[:3] if kind == "linear" else s
    assert getattr(lib, "stacklstm_%s_create" % kind)(ctypes.byref(h), *args, *tail) == OK
    return h


def t(n):
    return [0x100000 * (i + 1) for i in range(n)]


# name -> (operator, arguments after the handle; None in `may` where a pointer may be null)
def calls():
    return {"norm_forward": ("norm", [40, *t(3), 1e-5, *[0x900000 + 0x1000 * i for i in range(3)]], {2, 3, 6, 7}),
            "norm_backward": ("norm", [40, *t(8)], {3, 6, 7, 8}),
            "linear_forward": ("linear", [40, *t(6)], {3, 4, 6}),
            "linear_backward": ("linear", [40, *t(8)], {5, 6, 7, 8}),
            "distill_run": ("distill", [40, *t(4), 1.0, 0.5, 1.0, 0x900000, 0xA00000], {4, 8, 9}),
            "beam_lse": ("beam", t(2), set()),
            "beam_select": ("beam", t(7), {1, 3}),
            "beam_reorder": ("beam", t(9), {7, 8}),
            "beam_push": ("beam", t(8), {6, 7})}


@pytest.mark.parametrize("name", sorted(calls()))
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_calls_check_their_arguments(lib, name, dtype):
    kind, args, may = calls()[name]
    call = getattr(lib, "stacklstm_" + name)
    h = create(lib, kind, dtype)
    lib.fake_reset()
    assert call(h, *args) == OK and lib.stacklstm_op_last_error(h) == b""
    assert lib.fake_log()
    pointers = [i for i, a in enumerate(args) if isinstance(a, int) and a >= 0x100000]
    for i in pointers:
        lib.fake_reset()
        bad = list(args)
        bad[i] = None
        # (a null pre is refused for the activation of this layer alone)
        want = OK if i in may and not (name == "linear_backward" and i == 4) else ARG
        assert call(h, *bad) == want, i
        if want == ARG:
            assert lib.stacklstm_op_last_error(h) and not lib.fake_log()
        bad[i] = args[i] + 4
        lib.fake_reset()
        assert call(h, *bad) == ARG and b"aligned" in lib.stacklstm_op_last_error(h) and not lib.fake_log()
    for other in SIZES:
        if other != kind:
            o = create(lib, other, dtype)
            assert call(o, *args) == ARG
            lib.stacklstm_op_destroy(o)
    assert call(None, *args) == ARG
    lib.stacklstm_op_destroy(h)


@pytest.mark.parametrize("name", ["norm_forward", "norm_backward", "linear_forward", "linear_backward", "distill_run"])
def test_rows_outside_the_handles(lib, name):
    kind, args, _ = calls()[name]
    h = create(lib, kind)
    call = getattr(lib, "stacklstm_" + name)
    lib.fake_reset()
    assert call(h, 41, *args[1:]) == ARG and call(h, -1, *args[1:]) == ARG and not lib.fake_log()
    assert call(h, 0, *args[1:]) == OK and not lib.fake_log()  # no kernel for no rows
    lib.stacklstm_op_destroy(h)


@pytest.mark.parametrize("kind,clears", [("norm", 1), ("linear", 2), ("distill", 1), ("beam", 2)])
def test_a_new_handle_is_cleared_on_its_stream(lib, kind, clears):
    """The status word and the arrival counters, before a call on that stream can use them."""
    lib.fake_reset()
    h = create(lib, kind)
    assert lib.fake_calls() >= clears and lib.fake_unjoined(vp(USER)) == 0
    lib.stacklstm_op_destroy(h)


def test_numbers_are_checked(lib):
    h = create(lib, "norm")
    a = calls()["norm_forward"][1]
    for eps in (-1.0, float("nan")):
        assert lib.stacklstm_norm_forward(h, *a[:4], eps, *a[5:]) == ARG
    lib.stacklstm_op_destroy(h)
    h = create(lib, "distill")
    a = calls()["distill_run"][1]
    for tau, alpha in ((0.0, 0.5), (-1.0, 0.5), (float("nan"), 0.5), (float("inf"), 0.5), (1.0, -0.1), (1.0, 1.1), (1.0, float("nan"))):
        assert lib.stacklstm_distill_run(h, *a[:5], tau, alpha, *a[7:]) == ARG
    lib.stacklstm_op_destroy(h)


def test_tensors_that_must_differ(lib):
    h = create(lib, "beam")
    a = t(7)
    a[4] = a[2]
    assert lib.stacklstm_beam_select(h, *a) == ARG
    for old, new in ((1, 4), (2, 5), (3, 6)):
        a = t(9)
        a[new] = a[old]
        assert lib.stacklstm_beam_reorder(h, *a) == ARG
    lib.stacklstm_op_destroy(h)


@pytest.mark.parametrize("name", sorted(calls()))
@pytest.mark.parametrize("dtype,sizes", [(FP32, None), (BF16, None), (BF16, "odd")])
def test_a_call_that_fails_says_so_and_stays_on_its_stream(lib, name, dtype, sizes):
    kind, args, _ = calls()[name]
    odd = {"norm": (40, 23), "linear": (40, 23, 17, 2), "distill": (40, 23, 3), "beam": (5, 8, 2300, 7, 15)}
    h = create(lib, kind, dtype, odd[kind] if sizes else None)
    call = getattr(lib, "stacklstm_" + name)
    assert call(h, *args) == OK  # (the workspace is there)
    lib.fake_reset()
    assert call(h, *args) == OK
    n = lib.fake_calls()
    assert n >= 1 and all(line.split()[-1] == str(USER) for line in lib.fake_log().decode().splitlines())
    for k in range(n):
        lib.fake_reset()
        lib.fake_fail_at(k)
        assert call(h, *args) == CUDA, k
        assert b"stacklstm_" + name.encode() in lib.stacklstm_op_last_error(h)
    lib.fake_reset()
    assert lib.stacklstm_op_set_stream(h, OTHER) == OK and call(h, *args) == OK
    assert all(line.split()[-1] == str(OTHER) for line in lib.fake_log().decode().splitlines())
    lib.fake_reset()
    lib.stacklstm_op_destroy(h)


@pytest.mark.parametrize("kind,args,want", [
    ("norm", (0, 8, 0), ARG), ("norm", (4, 0, 0), ARG), ("norm", (4, 8, 2), ARG), ("norm", (4, 1 << 25, 0), UNSUPPORTED),
    ("linear", (0, 8, 8, 0, 0), ARG), ("linear", (4, 0, 8, 0, 0), ARG), ("linear", (4, 8, 0, 0, 0), ARG),
    ("linear", (4, 8, 8, 3, 0), ARG), ("linear", (4, 8, 8, 0, 5), ARG), ("linear", (4, 8, 8, 0, -1), ARG),
    ("linear", (4, 1 << 24, 8, 0, 0), UNSUPPORTED), ("distill", (0, 8, 1, 0), ARG), ("distill", (4, 0, 1, 0), ARG),
    ("distill", (4, 8, 0, 0), ARG), ("distill", (4, 8, 257, 0), UNSUPPORTED), ("beam", (0, 1, 1, 1, 1, 0), ARG),
    ("beam", (1, 0, 1, 1, 1, 0), ARG), ("beam", (1, 1, 0, 1, 1, 0), ARG), ("beam", (1, 1, 1, 0, 1, 0), ARG),
    ("beam", (1, 1, 1, 1, 0, 0), ARG), ("beam", (1, 65, 1, 1, 1, 0), UNSUPPORTED), ("beam", (1, 64, 1 << 25, 1, 1, 0), UNSUPPORTED),
    ("beam", (65536, 1, 1, 1, 1, 0), UNSUPPORTED)])
def test_create_rejects_bad_sizes(real, kind, args, want):
    h = vp(1)
    assert getattr(real, "stacklstm_%s_create" % kind)(ctypes.byref(h), *args, 0, None) == want
    assert h.value is None
    assert getattr(real, "stacklstm_%s_create" % kind)(None, *args, 0, None) == ARG


def test_null_handles(real):
    assert real.stacklstm_op_status(None) == ARG and real.stacklstm_op_set_stream(None, None) == ARG
    assert real.stacklstm_op_destroy(None) == OK and real.stacklstm_op_last_error(None) == b"null handle"


def test_norm_workspace(lib):
    """Nothing for wide rows until a backward wants their column sums, and those within a bound; all of
    it at create for rows that fit registers, so that no call allocates."""
    lib.cudaMalloc.argtypes = [ctypes.POINTER(vp), ctypes.c_size_t]

    def allocated(f):  # (the stand-in's addresses follow one another)
        a, b = vp(), vp()
        lib.cudaMalloc(ctypes.byref(a), 0)
        r = f()
        lib.cudaMalloc(ctypes.byref(b), 0)
        return r, b.value - a.value

    P = t(8)
    for dtype in (FP32, BF16):
        h, n = allocated(lambda: create(lib, "norm", dtype, (1 << 16, 1 << 24)))
        assert n < 1 << 20
        assert allocated(lambda: lib.stacklstm_norm_forward(h, 1 << 16, *P[:3], 1e-5, *P[3:6]))[1] < 1 << 20
        assert allocated(lambda: lib.stacklstm_norm_backward(h, 1 << 16, *P[:6], None, None))[1] < 1 << 20
        st, n = allocated(lambda: lib.stacklstm_norm_backward(h, 1 << 16, *P))
        assert st == OK and 8 << 24 <= n <= (4 << 30) + (1 << 20)
        lib.stacklstm_op_destroy(h)
        for N in (100, 1024, 4095, 4096):
            h, n = allocated(lambda: create(lib, "norm", dtype, (1 << 16, N)))
            assert 152 * 8 * N <= n < 11 << 20
            st, n = allocated(lambda: lib.stacklstm_norm_backward(h, 1 << 16, *P))
            assert st == OK and n < 1 << 20
            lib.stacklstm_op_destroy(h)
