"""What asap_xent_forward, asap_xent_backward and their Python forms refuse, all of it before the GPU is touched, and the
workspace sizes they ask for.  No GPU: the pointers below are numbers that are never followed."""
import ctypes as C

import pytest
import torch

from paper_1612_08608_gb300 import build


@pytest.fixture(scope="module")
def lib():
    build.build()
    from paper_1612_08608_gb300._lib import load_library
    return load_library()


BASE = dict(N=2, n=100, C=300, d=64, dtype=1, X=1 << 32, ldx=64, sx=6400, W=2 << 32, ldw=64, sw=19200, y=3 << 32, loss=4 << 32,
            lse=5 << 32, g=6 << 32, dX=7 << 32, lddx=64, sdx=6400, dW=8 << 32, lddw=64, sdw=19200, ws=9 << 32, size=1 << 30)


def _forward(lib, **change):
    a = {**BASE, **change}
    return lib.asap_xent_forward(a["N"], a["n"], a["C"], a["d"], a["dtype"], a["X"], a["ldx"], a["sx"], a["W"], a["ldw"],
                                 a["sw"], a["y"], a["loss"], a["lse"], a["ws"], a["size"], None)


def _backward(lib, **change):
    a = {**BASE, **change}
    return lib.asap_xent_backward(a["N"], a["n"], a["C"], a["d"], a["dtype"], a["X"], a["ldx"], a["sx"], a["W"], a["ldw"],
                                  a["sw"], a["y"], a["lse"], a["g"], a["dX"], a["lddx"], a["sdx"], a["dW"], a["lddw"],
                                  a["sdw"], a["ws"], a["size"], None)


BOTH = [(dict(N=0), b"N"), (dict(N=1025), b"N"), (dict(n=-1), b"n"), (dict(n=(1 << 24) + 1), b"n"), (dict(C=0), b"C"),
        (dict(C=(1 << 28) + 1), b"C"), (dict(d=0), b"d"), (dict(d=(1 << 20) + 1), b"d"),
        (dict(N=1, n=1 << 24, C=1 << 28), b"tiles"), (dict(dtype=0), b"BF16"), (dict(dtype=3), b"BF16"),
        (dict(X=None), b"NULL"), (dict(W=None), b"NULL"), (dict(y=None), b"NULL"), (dict(lse=None), b"NULL"),
        (dict(ws=None), b"NULL"), (dict(X=(1 << 32) + 8), b"16"), (dict(ldx=60), b"16"), (dict(ldx=68), b"16"),
        (dict(W=(2 << 32) + 2), b"16"), (dict(ldw=63), b"16"), (dict(sx=6404), b"16"), (dict(sx=6392), b"16"),
        (dict(sw=0), b"16"), (dict(sw=-19200), b"16"), (dict(size=1000), b"workspace"), (dict(ws=(9 << 32) + 128), b"workspace"),
        (dict(ws=(1 << 32) + 256), b"overlap")]


@pytest.mark.parametrize("change,word", BOTH + [(dict(loss=None), b"NULL"), (dict(y=(3 << 32) + 2), b"4 bytes"), (dict(lse=(5 << 32) + 1), b"4 bytes"), (dict(loss=(5 << 32) + 4), b"overlap"),
                                                (dict(lse=3 << 32), b"overlap")])
def test_forward_refuses(lib, change, word):
    assert _forward(lib, **change) == 1
    assert word in lib.asap_last_error(None)


@pytest.mark.parametrize("change,word", BOTH + [
    (dict(g=None), b"NULL"), (dict(g=(6 << 32) + 2), b"4 bytes"), (dict(dX=None, dW=None), b"neither"), (dict(dX=(7 << 32) + 8), b"16"), (dict(lddx=32), b"16"),
    (dict(sdx=0), b"16"), (dict(sdw=64), b"16"), (dict(lddw=65), b"16"), (dict(dX=1 << 32), b"overlap"),
    (dict(dW=(2 << 32) + 1600), b"overlap"), (dict(dW=(7 << 32) + 16), b"overlap"), (dict(dX=6 << 32), b"overlap")])
def test_backward_refuses(lib, change, word):
    assert _backward(lib, **change) == 1
    assert word in lib.asap_last_error(None)


def test_debug_entry_refuses(lib):
    for bad in ((-1, 0, 1), (3, 0, 1), (0, -1, 1), (0, 0, 0)):
        assert lib.asap_debug_xent(*bad) == 1 and b"asap_debug_xent" in lib.asap_last_error(None)


def test_workspace_sizes(lib):
    least, good = C.c_uint64(), C.c_uint64()
    import random
    r = random.Random(1)
    for _ in range(300):
        N, n, V, d = r.choice([1, 1, 2, 32]), int(2 ** r.uniform(0, 15)), int(2 ** r.uniform(0, 18)), int(2 ** r.uniform(0, 13))
        for back in (0, 1):
            assert lib.asap_xent_workspace(N, n, V, d, back, C.byref(least), C.byref(good)) == 0
            assert 0 < least.value <= good.value
            # a byte less is refused; the least itself is taken (here it ends at the missing device, or the pointers)
            call = _backward if back else _forward
            pad = (d + 7) // 8 * 8
            sizes = dict(N=N, n=n, C=V, d=d, ldx=pad, sx=n * pad, ldw=pad, sw=V * pad, lddx=pad, sdx=n * pad, lddw=pad,
                         sdw=V * pad, X=1 << 44, W=2 << 44, y=3 << 44, loss=4 << 44, lse=5 << 44, g=6 << 44, dX=7 << 44,
                         dW=8 << 44, ws=9 << 44)
            assert call(lib, size=least.value - 1, **sizes) == 1
            assert b"workspace" in lib.asap_last_error(None)
            if not torch.cuda.is_available():
                for size in (least.value, (least.value + good.value) // 2, good.value):
                    assert call(lib, size=size, **sizes) == 2, lib.asap_last_error(None)     # ASAP_ERR_CUDA
    assert lib.asap_xent_workspace(0, 1, 1, 1, 0, C.byref(least), None) == 1
    assert lib.asap_xent_workspace(1, 1, 1, 1, 0, None, None) == 1


def test_python_forms_refuse_what_they_cannot_pass_on(lib):
    from paper_1612_08608_gb300 import ops
    b = torch.bfloat16
    X, W, y = torch.zeros(4, 8, dtype=b), torch.zeros(5, 8, dtype=b), torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(4)
    for bad in (lambda: ops.softmax_xent(X, W, y),                                       # not on a GPU
                lambda: ops.softmax_xent(X, W[:, :7], y), lambda: ops.softmax_xent(X[None], W, y),
                lambda: ops.softmax_xent(X.float(), W.float(), y), lambda: ops.softmax_xent(X, W.half(), y),
                lambda: ops.softmax_xent(X, W, y.long()), lambda: ops.softmax_xent(X, W, y[:3]),
                lambda: ops.softmax_xent(X, W, y, loss=f.double()), lambda: ops.softmax_xent_grad(X, W, y, f, f[:3]),
                lambda: ops.softmax_xent_grad(X, W, y, f, f, dX=X[:3]), lambda: ops.softmax_xent_grad(X, W, y, f, f, dW=W.half()),
                lambda: ops.softmax_xent(X.t().contiguous().t(), W, y)):
        with pytest.raises(ValueError):
            bad()
