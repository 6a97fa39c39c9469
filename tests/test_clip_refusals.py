"""What asap_clip_grads, asap_sgd_clipped and their Python forms refuse: all of it before the GPU is touched.  No GPU:
the pointers below are numbers that are never followed."""
import ctypes as C

import pytest
import torch

from paper_1612_08608_gb300 import build

P = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    build.build()
    from paper_1612_08608_gb300._lib import load_library
    return load_library()


def _arrays(ptrs, numel, dtypes, groups=None):
    T = len(ptrs)
    return ((P * T)(*ptrs), (C.c_int64 * T)(*numel), (C.c_int32 * T)(*dtypes),
            None if groups is None else (C.c_int32 * T)(*groups))


def _clip(lib, grads=(0x10000,), out=(0x20000,), numel=(8,), dtypes=(0,), groups=None, n_groups=1, max_norm=1.0,
          norms=0x30000, ws=0x40000, size=1 << 20, count=None):
    g, n, t, k = _arrays(grads, numel, dtypes, groups)
    o = None if out is None else (P * len(out))(*out)
    return lib.asap_clip_grads(len(grads) if count is None else count, g, o, n, t, k, n_groups, max_norm, norms, ws, size,
                               None)


@pytest.mark.parametrize("change,word", [
    (dict(count=-1), b"count"), (dict(n_groups=0), b"n_groups"), (dict(n_groups=65537), b"n_groups"),
    (dict(norms=None), b"NULL"), (dict(ws=None), b"NULL"), (dict(grads=(None,)), b"NULL"), (dict(out=(None,)), b"NULL"),
    (dict(size=8), b"workspace"), (dict(ws=0x40008), b"workspace"), (dict(norms=0x30002), b"norms"),
    (dict(max_norm=0.0), b"max_norm"), (dict(max_norm=-1.0), b"max_norm"), (dict(max_norm=float("nan")), b"max_norm"),
    (dict(dtypes=(3,)), b"type"), (dict(dtypes=(-1,)), b"type"), (dict(groups=(1,)), b"group"), (dict(groups=(-1,)), b"group"),
    (dict(numel=(-1,)), b"count"), (dict(numel=((1 << 40) + 1,)), b"count"),
    (dict(grads=(0x10002,)), b"aligned"), (dict(out=(0x20001,), dtypes=(1,)), b"aligned"),
    (dict(out=(0x10004,)), b"overlap"),                                                  # shifted, not in place
    (dict(grads=(0x10000, 0x10010), out=(0x20000, 0x20010), numel=(8, 8), dtypes=(0, 0)), b"overlap"),   # outs meet
    (dict(grads=(0x10000, 0x20000), out=(0x20000, 0x30000), numel=(8, 8), dtypes=(0, 0)), b"overlap"),   # another's gradient
    (dict(grads=(0x10000, 0x10000), out=(0x10000, 0x10000), numel=(8, 8), dtypes=(0, 0)), b"overlap"),   # the same one twice
])
def test_clip_refuses(lib, change, word):
    assert _clip(lib, **change) == 1
    assert word in lib.asap_last_error(None)


def _sgd(lib, params=(0x10000,), copies=(0x50000,), ctypes=(1,), grads=(0x20000,), numel=(8,), dtypes=(1,), lr=0.1, l2=0.0,
         **kw):
    g, n, t, _ = _arrays(grads, numel, dtypes)
    p = None if params is None else (P * len(params))(*params)
    c = None if copies is None else (P * len(copies))(*copies)
    k = None if ctypes is None else (C.c_int32 * len(ctypes))(*ctypes)
    return lib.asap_sgd_clipped(len(grads), p, c, k, g, n, t, None, 1, 1.0, lr, l2, 0x30000, 0x40000, 1 << 20, None)


@pytest.mark.parametrize("change,word", [
    (dict(lr=0.0), b"lr"), (dict(lr=-1.0), b"lr"), (dict(l2=-1.0), b"l2"), (dict(lr=1.0, l2=1.0), b"lr*l2"),
    (dict(lr=float("nan")), b"lr"), (dict(params=None), b"NULL"), (dict(params=(None,)), b"NULL"),
    (dict(ctypes=(0,)), b"type"), (dict(ctypes=None), b"type"), (dict(copies=(0x50001,)), b"aligned"),
    (dict(params=(0x10002,)), b"aligned"), (dict(copies=(0x10010,)), b"overlap"), (dict(params=(0x20000,)), b"overlap"),
])
def test_sgd_refuses(lib, change, word):
    assert _sgd(lib, **change) == 1
    assert word in lib.asap_last_error(None)


def test_workspace_sizes(lib):
    v = C.c_uint64()
    assert lib.asap_clip_workspace(1, 1, C.byref(v)) == 0 and v.value > 0
    one = v.value
    assert lib.asap_clip_workspace(1, 65536, C.byref(v)) == 0 and v.value > one
    for k in (0, -1, 65537):
        assert lib.asap_clip_workspace(1, k, C.byref(v)) == 1
    assert lib.asap_clip_workspace(1, 1, None) == 1
    assert lib.asap_clip_workspace(-1, 1, C.byref(v)) == 1


def test_python_forms_refuse_what_they_cannot_pass_on(lib):
    from paper_1612_08608_gb300 import ops
    x = torch.zeros(4)
    for bad in (lambda: ops.clip_grads([]), lambda: ops.clip_grads([x]),                   # nothing; not on a GPU
                lambda: ops.clip_grads([x], out=[x, x]), lambda: ops.clip_grads([x], out=[torch.zeros(3)]),
                lambda: ops.clip_grads([x], out=[x.half()]), lambda: ops.sgd_step([x.half()], [x], 0.1),
                lambda: ops.sgd_step([], [], 0.1), lambda: ops.sgd_step([x], [x], 0.1, copies=[x])):
        with pytest.raises(ValueError):
            bad()
