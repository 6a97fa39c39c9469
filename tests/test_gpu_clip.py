"""Global gradient norms, clipping and the clipped SGD step (GPU) against their definitions in 64 bits.

Tolerances, in units u = 2^-24 (half a step of fp32): a sum of squares is off by at most about 18 u (the squares and at
most 16 additions in a row in fp32, the rest wider), so a norm by 9 u and its own rounding, 12 u here; a scale by one more
division, 14 u; an output by its own rounding besides, half a step of its type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F16_TINY = 2.0 ** -25            # half the smallest fp16 step


def _grads(sizes, dtypes, seed, offsets=None, scale=1.0):
    """Tensors of the given sizes; offsets: elements by which each is off a 256-byte boundary."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        o = offsets[i % len(offsets)] if offsets else 0
        x = torch.randn(n + o, generator=g, device="cuda") * scale
        out.append(x.to(getattr(torch, dtypes[i % len(dtypes)]))[o:])
    return out


def _want(grads, groups, n_groups, max_norm):
    sq = [0.0] * n_groups
    for g, k in zip(grads, groups):
        sq[k] += float(g.double().pow(2).sum())
    norms = [math.sqrt(v) for v in sq]
    return norms, [max_norm / v if v > max_norm else 1.0 for v in norms]


def _close(got, want, dtype, rel=14 * U):
    import torch
    tol = want.abs() * (rel + torch.finfo(dtype).eps / 2)
    if dtype == torch.float16:
        tol = tol + F16_TINY
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])


SHAPES = {
    "one element": [1],
    "one tensor": [5],
    "ends of a vector": [7, 8, 9, 15, 16, 17, 31, 33],
    "around a chunk": [16383, 16384, 16385, 16391, 32768, 32769],
    "empty among others": [0, 100, 0, 3, 0],
    "a large one": [3000001, 1, 70000],
    "more than one table": [1 + (i * 37) % 300 for i in range(1300)],
}


@pytest.mark.parametrize("dtypes", [["float32"], ["bfloat16"], ["float16"], ["bfloat16", "float32", "float16"]])
@pytest.mark.parametrize("name", SHAPES)
def test_clip_against_the_definition(name, dtypes):
    import torch

    from paper_1612_08608_gb300 import ops
    sizes = SHAPES[name]
    for offsets, G in (([0], 1), ([0, 1, 2, 3, 5, 7], min(3, len(sizes)))):
        grads = _grads(sizes, dtypes, seed=len(sizes) + G, offsets=offsets)
        groups = [(i * 7) % G for i in range(len(sizes))]                # not sorted
        for factor in (0.25, 4.0):                                        # clipped, and not
            max_norm = factor * math.sqrt(sum(sizes) / G)
            norms_w, scale = _want(grads, groups, G, max_norm)
            out = [torch.full_like(g, float("nan")) for g in grads]
            norms = ops.clip_grads(grads, max_norm, out=out, groups=groups, n_groups=G)
            got = norms.tolist()
            assert all(abs(a - b) <= 12 * U * b for a, b in zip(got, norms_w)), (got, norms_w)
            for o, g, k in zip(out, grads, groups):
                _close(o, g.double() * scale[k], g.dtype)
            # In place, on copies.  They lie at other addresses, by which elements are summed together: both norms
            # are within 12 u of the definition's, and may differ in their last bit.
            again = [g.clone() for g in grads]
            got = ops.clip_grads(again, max_norm, groups=groups, n_groups=G).tolist()
            assert all(abs(a - b) <= 12 * U * b for a, b in zip(got, norms_w)), (got, norms_w)
            for a, g, k in zip(again, grads, groups):
                _close(a, g.double() * scale[k], g.dtype)
            assert torch.equal(ops.clip_grads(grads, groups=groups, n_groups=G), norms)    # norms alone


@pytest.mark.parametrize("offsets", [[0], [1, 2, 3], [4, 8, 12]])
@pytest.mark.parametrize("gtype,ctype", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float16", "float16"),
                                         ("bfloat16", None), ("float32", "float16")])
def test_step_against_the_definition(gtype, ctype, offsets):
    import torch

    from paper_1612_08608_gb300 import ops
    sizes = [1, 7, 8, 23, 16384, 16399, 500003, 12]
    grads = _grads(sizes, [gtype], 3, offsets)
    w0 = _grads(sizes, ["float32"], 4, offsets)
    groups = [i % 2 for i in range(len(sizes))]
    copies = None
    if ctype:
        copies = _grads(sizes, [ctype], 5, offsets[::-1])
        copies[2] = None
    lr, l2 = float(np.float32(0.3)), float(np.float32(0.01))
    norms_w, scale = _want(grads, groups, 2, 300.0)
    assert min(scale) < 1.0
    w = [x.clone() for x in w0] if offsets == [0] else [x for x in _grads(sizes, ["float32"], 4, offsets)]
    keep = [g.clone() for g in grads]
    norms = ops.sgd_step(w, grads, lr, 300.0, l2=l2, copies=copies, groups=groups)
    assert all(abs(a - b) <= 12 * U * b for a, b in zip(norms.tolist(), norms_w))
    for i, k in enumerate(groups):
        keepw, step = (1.0 - lr * l2) * w0[i].double(), lr * scale[k] * grads[i].double()
        # the factor of w: two roundings and the product's; the step: the scale's 14 and the rate's; the result's
        tol = 4 * U * keepw.abs() + 16 * U * step.abs() + U * (keepw - step).abs()
        assert bool(((w[i].double() - (keepw - step)).abs() <= tol).all()), i
        if copies is not None and copies[i] is not None:
            assert torch.equal(copies[i], w[i].to(copies[i].dtype))
        assert torch.equal(grads[i], keep[i])


@pytest.mark.parametrize("value", [1e25, 3e-30, 1e-40])
def test_squares_that_leave_the_range_of_fp32(value):
    import torch

    from paper_1612_08608_gb300 import ops
    g = torch.full((40000,), value, device="cuda")
    g[5:30000] = 0.0
    norms_w, _ = _want([g], [0], 1, 1.0)
    got = ops.clip_grads([g]).item()
    assert abs(got - norms_w[0]) <= 12 * U * norms_w[0] + 2.0 ** -149
    out = [torch.empty_like(g)]
    ops.clip_grads([g], norms_w[0] / 2, out=out)
    _close(out[0], g.double() / 2, torch.float32, rel=14 * U + (2.0 ** -149) / abs(value))


def test_zero_gradients_and_empty_groups():
    import torch

    from paper_1612_08608_gb300 import ops
    g = [torch.zeros(100000, device="cuda"), torch.zeros(0, device="cuda"), torch.ones(4, device="cuda")]
    norms = ops.clip_grads(g, 0.5, groups=[4, 2, 0], n_groups=6)
    assert norms.tolist() == [2.0, 0.0, 0.0, 0.0, 0.0, 0.0]
    assert g[2].tolist() == [0.25] * 4 and not bool(g[0].any())
    assert ops.clip_grads([g[1]], 0.5).tolist() == [0.0]


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_not_finite(bad):
    import torch

    from paper_1612_08608_gb300 import ops
    g = [torch.ones(20000, device="cuda"), torch.ones(20000, device="cuda")]
    g[1][12345] = bad
    keep = [x.clone() for x in g]
    norms = ops.clip_grads(g, 1.0, groups=[0, 1])
    assert abs(norms[0].item() - math.sqrt(20000.0)) < 1e-4 and not math.isfinite(norms[1].item())
    assert torch.equal(torch.nan_to_num(g[1]), torch.nan_to_num(keep[1]))                       # not scaled
    w = [torch.ones(20000, device="cuda"), torch.ones(20000, device="cuda")]
    c = [x.bfloat16() * 0 for x in w]
    ops.sgd_step(w, keep, 0.1, 1.0, copies=c, groups=[0, 1])
    assert bool((w[0] < 1).all()) and bool((w[1] == 1).all()) and bool((c[1] == 0).all())       # no step for group 1


def test_a_scale_that_vanishes_is_still_a_scale():
    import torch

    from paper_1612_08608_gb300 import ops
    g, w = [torch.full((3000,), 1e12, device="cuda")], [torch.ones(3000, device="cuda")]
    out = [torch.full_like(g[0], float("nan"))]
    ops.clip_grads(g, 1e-38, out=out)                            # 1e-38 / 5e13 is 0 in fp32
    assert bool((out[0] == 0).all())
    ops.sgd_step(w, g, 0.5, 1e-38, l2=0.5)
    assert bool((w[0] == 0.75).all())                            # the shrink alone


def test_tensors_beyond_32_bit_offsets():
    import torch

    from paper_1612_08608_gb300 import ops
    n = 2 ** 31 + 70001
    flat = torch.empty(n + 3, dtype=torch.float16, device="cuda")
    for part in flat.split(2 ** 28):
        part.fill_(0.25)
    g = flat[3:]
    g[-1], g[2 ** 31], g[2 ** 31 - 1] = 100.0, 7.0, 5.0
    want = math.sqrt((n - 3) * 0.0625 + 1e4 + 49.0 + 25.0)
    norms = ops.clip_grads([g, torch.ones(5, device="cuda")], want / 4, groups=[0, 1])
    assert abs(norms[0].item() - want) <= 12 * U * want
    head = float(torch.tensor(0.0625, dtype=torch.float16))      # 0.25 / 4 to within a rounding
    for part in g.split(2 ** 28):
        assert float(part.min()) >= head * (1 - 2.0 ** -10) and int((part > head * (1 + 2.0 ** -10)).sum()) <= 3
    assert [float(g[i]) for i in (-1, 2 ** 31, 2 ** 31 - 1)] == [25.0, 1.75, 1.25]
    assert float(flat[2]) == 0.25                                # what lies before it


def test_many_groups_and_the_same_bits_twice():
    import torch

    from paper_1612_08608_gb300 import ops
    sizes = [1 + (i * 7919) % 5000 for i in range(2000)]
    grads = _grads(sizes, ["bfloat16"], 9)
    groups = [(i * 31) % 999 for i in range(2000)]
    norms_w, scale = _want(grads, groups, 1000, 20.0)
    out = [torch.empty_like(g) for g in grads]
    ws = torch.full((ops.clip_workspace(2000, 1000),), 255, dtype=torch.uint8, device="cuda")        # any contents
    norms = ops.clip_grads(grads, 20.0, out=out, groups=groups, n_groups=1000, workspace=ws)
    assert all(abs(a - b) <= 12 * U * b for a, b in zip(norms.tolist(), norms_w))
    for o, g, k in zip(out, grads, groups):
        _close(o, g.double() * scale[k], g.dtype)
    for _ in range(3):
        assert torch.equal(ops.clip_grads(grads, 20.0, out=out, groups=groups, n_groups=1000), norms)


@pytest.mark.parametrize("tensors", [3, 50, 700])                 # a small table, a large one, two
def test_streams_and_graphs(tensors):
    import torch

    from paper_1612_08608_gb300 import ops
    grads = _grads([70000, 3, 16385] + [1 + (i * 53) % 900 for i in range(tensors - 3)], ["bfloat16", "float32"], 11)
    out = [torch.empty_like(g) for g in grads]
    want = ops.clip_grads(grads, 5.0, out=out).clone()
    want_out = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in out:
            o.zero_()
        got = ops.clip_grads(grads, 5.0, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(out, want_out))
    # two graphs on one workspace, replayed in turn; inputs change between replays
    ws = torch.empty(ops.clip_workspace(tensors), dtype=torch.uint8, device="cuda")
    graphs, results = [], []
    for max_norm in (5.0, 50.0):
        o = [torch.empty_like(g) for g in grads]
        n = torch.empty(1, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.clip_grads(grads, max_norm, out=o, norms=n, workspace=ws)
        graphs.append(g)
        results.append((max_norm, o, n))
    for turn in range(3):
        for g in grads:
            g.mul_(1.0 + turn)
        for g, (max_norm, o, n) in zip(graphs, results):
            g.replay()
            ref = [torch.empty_like(x) for x in grads]
            assert torch.equal(ops.clip_grads(grads, max_norm, out=ref), n)
            assert all(torch.equal(a, b) for a, b in zip(o, ref))
