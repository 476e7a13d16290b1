"""CPU: which kernels a gate or weight-gradient call launches: csrc/gate.cu and
csrc/tile_host.cu linked against a runtime that launches nothing and notes what it
was asked for (fake_tiles_runtime.cpp, fake_tiles.cu).  152 SMs."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_05613_gb300 import build as nb
from paper_2606_05613_gb300 import native as bk
from tile_shapes import BACKWARD, FORWARD, WGRAD, rows

HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16 = bk.BKMOO_F32, bk.BKMOO_BF16
P = 1 << 40                       # an aligned address, never touched


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    d = tmp_path_factory.mktemp("fake_tiles")
    objs = []
    for src in (os.path.join(nb.CSRC, "gate.cu"), os.path.join(nb.CSRC, "tile_host.cu"),
                os.path.join(HERE, "fake_tiles.cu"), os.path.join(HERE, "fake_tiles_runtime.cpp")):
        objs.append(str(d / (os.path.basename(src) + ".o")))
        subprocess.run([nb.nvcc()] + nb.ARCH + ["-I", nb.INCLUDE, "-I", nb.CSRC, "-std=c++17", "-Xcompiler", "-fPIC",
                                                "--expt-relaxed-constexpr", "-c", src, "-o", objs[-1]], check=True)
    so = str(d / "libfaketiles.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", so] + objs + ["-lpthread"], check=True)
    lib = ctypes.CDLL(so)
    lib.fake_notes.restype = ctypes.c_char_p
    return lib


def _launches(lib, call, *args):
    """(return code, kernels launched) of a call."""
    lib.fake_reset(0)
    code = call(*args)
    return code, [n for n in lib.fake_notes().decode().split() if not n.startswith("room:")]


def _up(n):
    return (n + 7) // 8 * 8


def _even(T, K):
    return (ctypes.c_int64 * (K + 1))(*[T * k // K for k in range(K + 1)])


def _places(K, at):
    return (ctypes.c_void_p * K)(*[P + (k << 36) + at for k in range(K)])


I64 = ctypes.c_int64


def _wgrad(lib, T, M, N, K, dtype, at=0, accumulate=0, rows=None):
    return _launches(lib, lib.bkmoo_language_wgrad, ctypes.c_void_p(P), I64(_up(M)), ctypes.c_void_p(P), I64(_up(N)),
                     I64(T), I64(M), I64(N), K, rows or _even(T, K), _places(K, at), dtype, accumulate, None)


def _backward(lib, T, D, F, K, dtype, at=0, accumulate=0, dx=True, rows=None):
    return _launches(lib, lib.bkmoo_gate_backward, ctypes.c_void_p(P), I64(_up(F)), ctypes.c_void_p(P), ctypes.c_void_p(P),
                     I64(_up(F)), ctypes.c_void_p(P), I64(_up(D)), ctypes.c_void_p(P), ctypes.c_void_p(P), I64(_up(D)),
                     I64(T), I64(D), I64(F), 0, K, rows or _even(T, K), ctypes.c_void_p(P if dx else 0), I64(_up(D)),
                     _places(K, at), _places(K, at), dtype, accumulate, ctypes.c_void_p(P), ctypes.c_size_t(1 << 50), None)


# bf16 gradients that are not whole or not aligned, from a few rows in many languages to
# more than the card holds
TURNED = [(2174, 288, 2450, 8), (300, 288, 2450, 8), (700, 650, 534, 16), (2100, 900, 1030, 4), (90, 100, 2451, 2),
          (4000, 1031, 1533, 2), (649, 6178, 534, 16), (4243, 6716, 6034, 4), (16384, 8191, 8190, 1), (8192, 8192, 8192, 16)]


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("T,M,N,K", TURNED)
def test_unaligned_bf16_gradients_take_at_most_128_columns(fake, T, M, N, K, accumulate):
    """The kernels of 256 columns that write such gradients do not exist: one of them ended
    in a fault of the GPU whose cause was not found."""
    allowed = {"1x64-turned", "1x128-turned"}
    code, names = _wgrad(fake, T, M, N, K, BF16, at=2 if N % 32 == 0 else 0, accumulate=accumulate)
    assert code == 0 and len(names) == 1 and names[0][len("weight-"):] in allowed
    for dx in (False, True):
        code, names = _backward(fake, T, N, M, K, BF16, at=2 if N % 32 == 0 else 0, accumulate=accumulate, dx=dx)
        assert code == 0 and names[0] == "pass" and len(names) == 2 and names[1][len("both-"):] in allowed


@pytest.mark.parametrize("T,M,N,K,at,modes", [
    (1024, 512, 544, 4, 0, ("sums", "sums-added", "plain", "added")),
    (1024, 512, 545, 4, 0, ("sums-turned", "sums-turned-added", "turned", "turned")),
    (1024, 512, 544, 4, 4, ("sums-turned", "sums-turned-added", "turned", "turned")),
    (700, 1, 300, 2, 0, ("sums-turned", "sums-turned-added", "turned", "turned")),
])
def test_kernels_that_add_are_kernels_of_their_own(fake, T, M, N, K, at, modes):
    """What fetches ahead the gradients that it adds to costs nothing where nothing is
    added; bf16 gradients that are turned have one kernel for both, without it."""
    want = iter(modes)
    for dtype in (F32, BF16):
        for accumulate in (0, 1):
            mode = next(want)
            code, names = _wgrad(fake, T, M, N, K, dtype, at=at, accumulate=accumulate)
            assert code == 0 and [n.split("-", 2)[2] for n in names] == [mode]
            code, names = _backward(fake, T, N, M, K, dtype, at=at, accumulate=accumulate)
            assert code == 0 and [n.split("-", 2)[2] for n in names[1:]] == [mode]


def test_status_copy_needs_a_place(fake):
    """(the calls' refusals, and that a copy neither launches nor clears)"""
    assert fake.bkmoo_op_status_copy(None, None) == bk.BKMOO_ERR_INVALID
    assert fake.bkmoo_op_status_copy(None, ctypes.c_void_p(P + 2)) == bk.BKMOO_ERR_INVALID
    assert _launches(fake, fake.bkmoo_op_status_copy, None, ctypes.c_void_p(P)) == (0, [])


def test_every_launch_asks_for_its_shared_memory(fake):
    """A kernel's limit on shared memory belongs to a context, which a cudaDeviceReset
    between two calls replaces: it is raised for every launch, whatever ran before."""
    for _ in range(2):
        for T, M, N, K in TURNED + [(8192, 2048, 8192, 4), (64, 256, 256, 2)]:
            for dtype in (F32, BF16):
                for accumulate in (0, 1):
                    code, names = _wgrad(fake, T, M, N, K, dtype, accumulate=accumulate)
                    notes = fake.fake_notes().decode().split()
                    assert code == 0 and notes == ["room:" + names[0], names[0]]


def _bounds(T, K):
    return (ctypes.c_int64 * (K + 1))(*rows(T, K))


@pytest.mark.parametrize("T,D,F,shape", FORWARD)
def test_sizes_of_the_forward_tests(fake, T, D, F, shape):
    v = ctypes.c_void_p(P)
    code, names = _launches(fake, fake.bkmoo_gate_forward, v, I64(_up(D)), v, v, I64(_up(D)), I64(T), I64(D), I64(F), 0,
                            v, I64(_up(F)), v, v, I64(_up(F)), None)
    assert (code, names) == (0, ["gate-%s-plain" % shape])


@pytest.mark.parametrize("call,T,A,B,K,aligned,odd,sums",
                         [("both",) + c for c in BACKWARD] + [("weight",) + c for c in WGRAD])
def test_sizes_of_the_gradient_tests(fake, call, T, A, B, K, aligned, odd, sums):
    run = _backward if call == "both" else _wgrad
    for accumulate in (0, 1):
        for dtype, at, shape, mode in ((BF16, 0, aligned, ("plain", "added")[accumulate]), (BF16, 6, odd, "turned"),
                                       (F32, 0, sums, ("sums", "sums-added")[accumulate]),
                                       (F32, 12, sums, ("sums-turned", "sums-turned-added")[accumulate])):
            code, names = run(fake, T, A, B, K, dtype, at=at, accumulate=accumulate, rows=_bounds(T, K))
            assert code == 0 and names[-1] == "%s-%s-%s" % (call, shape, mode)


def test_kernels_of_the_self_test(fake):
    for what, names in ((0, ["pass"]), (1, ["gate-1x256-plain"]), (2, ["gate-2x256-plain"])):
        assert _launches(fake, fake.bkmoo_selftest_give_up, what, None) == (0, names)
    for bad in (-1, 3):
        assert _launches(fake, fake.bkmoo_selftest_give_up, bad, None) == (bk.BKMOO_ERR_INVALID, [])
