"""Large-vocabulary cross entropy and its gradients (GPU) against their definitions in 64 bits.

Tolerances.  Products of 16-bit values are exact in fp32.  A logit is summed in steps of 16 products: each adds at most one
step (2^-23) of the sum of the products' magnitudes A, so z is off by tz = (d / 16 + 8) 2^-23 A.  lse moves by as much as the
z do, and by 2^-21 of its size and of 1 for exp2, log and their arguments.  R is off by half a step of its type and,
through p, by 3 times what z and lse are off; dX and dW sum it in steps of 16 again and are rounded once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _inputs(N, n, C, d, dtype, seed, pad=0, label=6.0, drop=0.0):
    """X, W, y, g: views in rows of d rounded up to 8, and `pad` more groups of 8."""
    import torch
    t = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rows(r, scale):
        ld = (d + 7) // 8 * 8 + 8 * pad
        x = torch.full((N, r, ld), float("nan"), device="cuda", dtype=t)      # what lies between rows is not read
        x[..., :d] = (torch.randn((N, r, d), generator=gen, device="cuda") * scale).to(t)
        return x[..., :d]
    X, W = rows(n, 1.0), rows(C, d ** -0.5)
    y = torch.randint(0, C, (N, n), generator=gen, device="cuda")
    X += (label * torch.rand((N, n, 1), generator=gen, device="cuda") *
          W[torch.arange(N, device="cuda")[:, None], y].float()).to(t)
    y = torch.where(torch.rand((N, n), generator=gen, device="cuda") < drop, torch.full_like(y, -100), y).to(torch.int32)
    g = torch.randn((N, n), generator=gen, device="cuda") / n
    return X, W, y, g


def _check(X, W, y, g, loss, lse, dX=None, dW=None, few=False):
    import torch
    N, n, d = X.shape
    C, eps = W.shape[1], torch.finfo(X.dtype).eps
    tiny = 2.0 ** -25 if X.dtype == torch.float16 else 0.0
    for i in range(N):
        rows = torch.nonzero((y[i] >= 0) & (y[i] < C)).flatten()
        out = torch.ones(n, dtype=torch.bool, device="cuda")
        out[rows] = False
        assert bool((lse[i][out] == 0).all())
        if dX is not None:
            assert bool((dX[i][out] == 0).all())
        x, w, yy = X[i][rows].double(), W[i].double(), y[i][rows].long()
        z = x @ w.T
        tz = (d / 16 + 8) * 2.0 ** -23 * ((x.abs() @ w.abs().T).max() if len(rows) else 0.0)
        want = torch.logsumexp(z, dim=1)
        tl = tz + 2.0 ** -21 * (want.abs() + 1)
        assert bool(((lse[i][rows] - want).abs() <= tl).all()), (lse[i][rows] - want).abs().max()
        wl = want - z[torch.arange(len(rows)), yy]
        assert bool(((loss[i][rows] - wl).abs() <= tl + tz).all()), (loss[i][rows] - wl).abs().max()
        if dX is None and dW is None:
            continue
        p = torch.exp(z - want[:, None])
        hot = torch.zeros_like(p)
        hot[torch.arange(len(rows)), yy] = 1.0
        gg = g[i][rows].double()[:, None]
        R, A = gg * (p - hot), gg.abs() * (p + hot)
        # a worker of 32 labels or fewer has R in two terms, each rounded: what `few` asks for
        half = eps * eps / 4 if few and len(rows) <= 32 else eps / 2
        off = half + 3 * (float(tz) + 2.0 ** -21 * (1 + float(want.abs().max()) if len(rows) else 0.0))
        small = float(gg.abs().max()) * 2.0 ** -38 if len(rows) and X.dtype == torch.float16 else 0.0
        if dX is not None:
            dx = R @ w
            tol = (off + (C / 16 + 16) * 2.0 ** -23) * (A @ w.abs()) + small * w.abs().sum(dim=0) + eps / 2 * dx.abs() + tiny
            assert bool(((dX[i][rows] - dx).abs() <= tol).all()), ((dX[i][rows] - dx).abs() / tol).max()
        if dW is not None:
            dw = R.T @ x
            tol = (off + (n / 16 + 16) * 2.0 ** -23) * (A.T @ x.abs()) + small * x.abs().sum(dim=0) + eps / 2 * dw.abs() + tiny
            assert bool(((dW[i] - dw).abs() <= tol).all()), ((dW[i] - dw).abs() / tol).max()


def _run(X, W, y, g, **kw):
    from paper_1612_08608_gb300 import ops
    loss, lse = ops.softmax_xent(X, W, y)
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, **kw)
    return loss, lse, dX, dW


SIZES = [(1, 1, 1, 1), (1, 1, 2, 8), (1, 1, 1000, 64), (1, 3, 257, 24), (2, 127, 300, 72), (1, 128, 256, 256),
         (1, 129, 512, 192), (3, 256, 130, 264), (1, 257, 1000, 320), (1, 64, 20000, 128), (1, 700, 2049, 520),
         (4, 300, 10, 256), (1, 1500, 777, 1100)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d", SIZES)
def test_loss_and_gradients(N, n, C, d, dtype):
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=N + n + C + d)
    _check(X, W, y, g, *_run(X, W, y, g))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d", [(1, 5, 33, 7), (1, 300, 600, 100), (2, 130, 515, 333), (1, 1025, 300, 65)])
def test_odd_sizes_in_padded_rows(N, n, C, d, dtype):
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=d, pad=3)
    _check(X, W, y, g, *_run(X, W, y, g))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d,pad", [(1, 1, 50001, 256, 0), (1, 2, 3000, 1001, 2), (3, 3, 999, 8, 0), (2, 4, 4099, 777, 1),
                                         (300, 1, 17, 40, 0), (1, 4, 40000, 2056, 0), (1, 5, 40000, 72, 0), (1, 1, 3, 24577, 0),
                                         (1, 1, 50, 20480, 0), (1, 4, 50, 5120, 0), (1, 1, 50, 24576, 0), (1, 2, 50, 12288, 0)])
def test_few_rows(N, n, C, d, pad, dtype):
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=C, pad=pad)
    y[0, n - 1] = C - 1
    _check(X, W, y, g, *_run(X, W, y, g))
    if n > 1:
        y[0, 0], y[N - 1, 1] = -5, -1                           # and rows without a label among them
        X[0, 0] = float("nan")
        _check(X, W, y, g, *_run(X, W, y, g))


def test_infinite_logits():
    import torch

    from paper_1612_08608_gb300 import ops
    for n in (2, 40):
        X, W, y, g = _inputs(1, n, 700, 64, "bfloat16", seed=2)
        ref = ops.softmax_xent(X, W, y)[1]
        y.fill_(300)
        X[0, 0, 0] = 1.0
        W[0, 5:9] = 0.0
        W[0, 5:9, 0] = float("-inf")                            # a masked class: exp of it is 0, where x_0 > 0
        X[0, 1:, 0] = X[0, 1:, 0].abs() + 0.5
        loss, lse = ops.softmax_xent(X, W, y)
        z = X[0].double() @ torch.where(torch.isinf(W[0]), 0.0, W[0].double()).T
        z[:, 5:9] = float("-inf")
        want = torch.logsumexp(z, 1)
        assert bool(((lse[0] - want).abs() <= 1e-4).all())      # 64 products of a few units, 2^-23 each
        W[0, 11, 0] = float("inf")                              # an infinite one leaves no finite loss
        loss, lse = ops.softmax_xent(X, W, y)
        assert not bool(torch.isfinite(loss).any())
        W[0, 11, 0] = float("nan")
        assert bool(torch.isnan(ops.softmax_xent(X, W, y)[1]).all())
        W[:] = 0.0
        W[0, :, 0] = float("-inf")                              # nothing is left of the vocabulary
        assert not bool(torch.isfinite(ops.softmax_xent(X, W, y)[0]).any())


@pytest.mark.parametrize("drop", [0.3, 0.97, 1.0])
@pytest.mark.parametrize("N,n,C,d", [(1, 40, 100, 64), (3, 600, 900, 136), (2, 1111, 300, 77)])
def test_rows_without_a_label(N, n, C, d, drop):
    import torch
    X, W, y, g = _inputs(N, n, C, d, "bfloat16", seed=n, drop=drop)
    if N > 1:
        y[1] = -1                                               # a worker with none
    for bad in (float("nan"), float("inf"), 3.0e38):
        X[y < 0] = bad                                          # nothing of these rows may show
        g[y < 0] = float("nan")
        _check(X, W, y, g, *_run(X, W, y, g))


def test_labels_out_of_range_make_the_loss_nan():
    import torch
    X, W, y, g = _inputs(1, 50, 100, 64, "bfloat16", seed=1)
    y[0, 7], y[0, 8] = 100, 2 ** 31 - 1
    loss, lse, dX, dW = _run(X, W, y, g)
    assert bool(torch.isnan(loss[0, 7:9]).all()) and int(torch.isnan(loss).sum()) == 2
    _check(X, W, y, g, loss, lse, dX, dW)


@pytest.mark.parametrize("N,n,C,d", [(1, 300, 3000, 200), (1, 20, 5000, 64), (2, 513, 1100, 320), (1, 2500, 1025, 3000)])
def test_pieces_of_the_vocabulary(N, n, C, d):
    import torch

    from paper_1612_08608_gb300 import ops
    X, W, y, g = _inputs(N, n, C, d, "bfloat16", seed=C, drop=0.2)
    least, good = ops.xent_workspace(N, n, C, d, grad=True)
    loss, lse = ops.softmax_xent(X, W, y)
    seen = []
    for size in (least, least + 300000, good, good + 12345):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")        # any contents
        dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
        _check(X, W, y, g, loss, lse, dX, dW)
        again = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
        assert torch.equal(again[0], dX) and torch.equal(again[1], dW)         # the same bits
        seen.append(dW)
    assert all(torch.equal(s, seen[0]) for s in seen)           # dW does not depend on the pieces
    only_x = ops.softmax_xent_grad(X, W, y, lse, g, need_dW=False)
    only_w = ops.softmax_xent_grad(X, W, y, lse, g, need_dX=False)
    assert only_x[1] is None and only_w[0] is None and torch.equal(only_w[1], seen[0])
    _check(X, W, y, g, loss, lse, only_x[0], only_w[1])


def test_large_logits_and_confident_rows():
    import torch
    X, W, y, g = _inputs(1, 200, 1000, 128, "bfloat16", seed=3, label=60.0)
    W *= 8.0                                                   # |z| in the hundreds: exp overflows without the maximum
    X[0, 5] = 0                                                # all logits alike
    loss, lse, dX, dW = _run(X, W, y, g)
    assert bool(torch.isfinite(loss).all())
    _check(X, W, y, g, loss, lse, dX, dW)


@pytest.mark.parametrize("scale", [1e-30, 1e-9, 1.0, 1e30])
def test_fp16_residuals_keep_their_precision_at_any_scale(scale):
    import torch
    X, W, y, g = _inputs(1, 96, 4000, 64, "float16", seed=5)
    g = torch.rand_like(g).add_(0.5).mul_(scale)
    W = (W.float() * min(1.0, 1e-26 / scale * 1e26 if scale > 1 else 1.0)).half()
    from paper_1612_08608_gb300 import ops
    _, lse = ops.softmax_xent(X, W, y)
    if scale > 1:                                              # gradients beyond fp16 become infinite, not wrong
        dX, dW = ops.softmax_xent_grad(X, W, y, lse, g)
        assert bool(torch.isinf(dW[0, y[0].long()]).any())
        return
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g)
    loss = torch.zeros_like(g)
    _check(X, W, y, g, ops.softmax_xent(X, W, y)[0], lse, dX, dW)


def test_gradient_against_differences():
    # d loss / dX along a direction, by a central difference of the 64-bit loss at X +- h u: exact to O(h^2)
    import torch
    X, W, y, g = _inputs(1, 64, 500, 96, "bfloat16", seed=8)
    _, _, dX, dW = _run(X, W, y, g)

    def f(x, w):
        z = x @ w.T
        return float((g[0].double() * (torch.logsumexp(z, 1) - z[torch.arange(64), y[0].long()])).sum())
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, h = X[0].double(), W[0].double(), 1e-4
    for t, grad in ((x, dX[0]), (w, dW[0])):
        u = torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64)
        step = (f(x + h * u, w) - f(x - h * u, w)) if t is x else (f(x, w + h * u) - f(x, w - h * u))
        got = float((grad.double() * u).sum())
        # half a step of bf16 in R and in the result, on every product, and the difference's own error
        tol = 2 * 2.0 ** -8 * float((grad.double().abs() * u.abs()).sum()) + 1e-5
        assert abs(step / (2 * h) - got) <= tol, (step / (2 * h), got, tol)


def test_no_rows():
    import torch

    from paper_1612_08608_gb300 import ops
    X = torch.zeros((2, 0, 64), dtype=torch.bfloat16, device="cuda")
    W = torch.ones((2, 30, 64), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    loss, lse = ops.softmax_xent(X, W, y)
    dW = torch.full_like(W, float("nan"))
    dX, _ = ops.softmax_xent_grad(X, W, y, lse, lse.clone(), dW=dW)
    assert loss.shape == (2, 0) and dX.shape == X.shape and bool((dW == 0).all())


def test_what_lies_around_the_outputs_is_left_alone():
    import torch

    from paper_1612_08608_gb300 import ops
    X, W, y, g = _inputs(2, 70, 300, 100, "bfloat16", seed=4, drop=0.3)
    _, lse = ops.softmax_xent(X, W, y)
    bx = torch.full((2, 73, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    bw = torch.full((2, 310, 120), 7.0, dtype=torch.bfloat16, device="cuda")
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, dX=bx[:, :70, :100], dW=bw[:, :300, :100])
    ref = ops.softmax_xent_grad(X, W, y, lse, g)
    assert torch.equal(dX, ref[0]) and torch.equal(dW, ref[1])
    assert bool((bx[:, 70:] == 7).all()) and bool((bx[:, :, 100:] == 7).all())
    assert bool((bw[:, 300:] == 7).all()) and bool((bw[:, :, 100:] == 7).all())


def test_a_confident_row_with_huge_logits_has_no_loss():
    # logits of some 1e5: the tensor cores' sums are off by tenths, the label's exact logit is not
    import torch

    from paper_1612_08608_gb300 import ops
    for n in (1, 30):
        X, W, y, g = _inputs(1, n, 400, 512, "bfloat16", seed=n)
        y[0] = torch.arange(n, device="cuda").to(torch.int32)
        X[0] = W[0, :n] * 512
        W[0] *= 512
        loss, lse = ops.softmax_xent(X, W, y)
        z = X[0].double() @ W[0].double().T
        own = z[torch.arange(n), y[0].long()]
        other = z.scatter(1, y[0].long()[:, None], float("-inf")).max()
        assert bool((own > 1e5).all()) and float(other) < float(own.min()) - 1e4
        assert bool(((lse[0] - own).abs() <= 2.0 ** -22 * own).all())
        assert bool((loss[0].abs() <= 2.0 ** -21 * own).all())


def test_heads_beyond_32_bit_offsets():
    # 600,000 classes of 4096: 2.46e9 elements, 4.9 GB each of W and dW
    import torch

    from paper_1612_08608_gb300 import ops
    C, d = 600000, 4096
    gen = torch.Generator(device="cuda").manual_seed(1)
    W = torch.empty((1, C, d), dtype=torch.bfloat16, device="cuda")
    for part in W[0].split(50000):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") / 64)
    edge = 2 ** 31 // d
    for n in (3, 40):
        X = torch.randn((1, n, d), generator=gen, device="cuda").bfloat16()
        y = torch.randint(0, C, (1, n), generator=gen, device="cuda").to(torch.int32)
        y[0, 0], y[0, 1], y[0, 2] = C - 1, edge, edge - 1
        g = torch.full((1, n), 1.0 / n, device="cuda")
        loss, lse, dX, dW = _run(X, W, y, g)
        z = torch.cat([X[0].double() @ part.double().T for part in W[0].split(50000)], dim=1)
        want = torch.logsumexp(z, 1)
        tol = (d / 16 + 8) * 2.0 ** -23 * 60 + 2.0 ** -18        # magnitudes of a logit's products: 4096 / 64 x 0.64
        assert bool(((lse[0] - want).abs() <= tol).all())
        assert bool(((loss[0] - (want - z[torch.arange(n), y[0].long()])).abs() <= 2 * tol).all())
        r = torch.exp(z - want[:, None])
        r[torch.arange(n), y[0].long()] -= 1.0
        r /= n
        rows = torch.cat([torch.arange(300), torch.arange(edge - 200, edge + 200), torch.arange(C - 300, C)]).cuda()
        dw, mag = r[:, rows].T @ X[0].double(), r[:, rows].abs().T @ X[0].double().abs()
        assert bool(((dW[0, rows] - dw).abs() <= (2.0 ** -8 + 4 * tol) * mag + 2.0 ** -8 * dw.abs()).all())
        dx = sum(r[:, i:i + 50000] @ W[0, i:i + 50000].double() for i in range(0, C, 50000))
        mag = sum(r[:, i:i + 50000].abs() @ W[0, i:i + 50000].double().abs() for i in range(0, C, 50000))
        assert bool(((dX[0] - dx).abs() <= (2.0 ** -8 + 4 * tol + C / 16 * 2.0 ** -23) * mag + 2.0 ** -8 * dx.abs()).all())
        del z, r, dX, dW


@pytest.mark.parametrize("kernel,tile", [(0, 0), (0, 1), (1, 0), (1, 1), (2, 0), (2, 1), (2, 2)])
@pytest.mark.parametrize("size", ["direct", "splits"])
def test_a_wait_that_runs_out(kernel, tile, size):
    # One CTA copies nothing from a tile on: the waits that depend on them end after 20 ms, the results say so, and the
    # next calls are whole.
    import torch

    from paper_1612_08608_gb300 import ops
    from paper_1612_08608_gb300._lib import load_library
    lib = load_library()
    # the first cluster of 76 has two tiles of logits and of R, and two of dX, then dW's; or three, and one of dX
    N, n, C, d = (8, 500, 1500, 1280) if size == "direct" else (1, 500, 30000, 512)
    X, W, y, g = _inputs(N, n, C, d, "bfloat16", seed=kernel, drop=0.1)
    _, lse = ops.softmax_xent(X, W, y)
    # (enough for one piece: of a narrow one a cluster would have a tile at most)
    ws = torch.empty(max(ops.xent_workspace(N, n, C, d, grad=k)[1] for k in (False, True)), dtype=torch.uint8, device="cuda")
    assert lib.asap_debug_xent(kernel, tile, 20_000_000) == 0
    if kernel == 0:
        loss, bad = ops.softmax_xent(X, W, y, workspace=ws)
        assert bool(torch.isnan(loss[y >= 0]).all()) and bool(torch.isnan(bad[y >= 0]).all())
    else:
        dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
        assert bool(torch.isnan(dX).any()) or bool(torch.isnan(dW).any())
    assert int(ws[:4].view(torch.int32)) == 4                                  # ASAP_ERR_TIMEOUT
    loss, lse = ops.softmax_xent(X, W, y, workspace=ws)
    assert int(ws[:4].view(torch.int32)) == 0
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
    assert int(ws[:4].view(torch.int32)) == 0
    _check(X, W, y, g, loss, lse, dX, dW)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d", [(1, 63, 3000, 1160), (1, 64, 41000, 520), (3, 65, 700, 1025), (5, 33, 1300, 577),
                                     (2, 17, 257, 2056), (20, 40, 300, 1000), (40, 64, 515, 513), (1, 1, 300, 40),
                                     (1, 2, 9000, 100), (76, 3, 60, 200), (3, 300, 700, 328),
                                     (1, 32, 41000, 264), (20, 32, 300, 1001), (20, 31, 300, 1000), (1, 33, 2000, 72)])
def test_short_tiles(N, n, C, d, dtype):
    # up to 32 rows with a label in every worker, or 64, just above, and above in one worker alone
    from paper_1612_08608_gb300 import ops
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=n)
    _check(X, W, y, g, *_run(X, W, y, g), few=True)
    if N > 1:
        y[1:, 1::2] = -100
        X[1:, 1::2] = float("inf")
        if n > 200:
            y[0, 33:], y[1, :240] = -100, -100                  # 33 and then 32, 30 and 150 of a label
        _check(X, W, y, g, *_run(X, W, y, g), few=True)
        y[0, 0] = -1
        _check(X, W, y, g, *_run(X, W, y, g), few=True)
    import torch
    ws = torch.empty(ops.xent_workspace(N, n, C, d, grad=True)[0], dtype=torch.uint8, device="cuda")     # pieces
    _check(X, W, y, g, *_run(X, W, y, g, workspace=ws), few=True)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d", [(1, 800, 10, 4096), (1, 40, 50, 4090), (6, 300, 300, 1024), (1, 300, 9500, 1100),
                                     (2, 3, 14, 2056), (1, 300, 9800, 1100), (1, 6, 10, 1023)])
def test_long_sums_of_few_classes(N, n, C, d, dtype):
    # Where a cluster has one tile at most, sums over 1024 features and more come in two parts; 9800 classes are too many.
    import torch
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=C + d, drop=0.2)
    loss, lse, dX, dW = _run(X, W, y, g)
    _check(X, W, y, g, loss, lse, dX, dW)
    if d >= 1024 and C < 9800:
        # 2^-23 of a sum lost by a step is what _check allows to both parts together: here to each, over half the steps
        for i in range(N):
            rows = torch.nonzero(y[i] >= 0).flatten()
            x, w = X[i][rows].double(), W[i].double()
            z = x @ w.T
            want = torch.logsumexp(z, dim=1)
            tl = (d / 32 + 8) * 2.0 ** -23 * float((x.abs() @ w.abs().T).max()) + 2.0 ** -21 * (want.abs() + 1)
            assert bool(((lse[i][rows] - want).abs() <= tl).all())


@pytest.mark.parametrize("n", [1, 2, 5, 40, 300])
@pytest.mark.parametrize("top", [50.25, 100.5, 129.0, 201.0])
def test_a_certain_row_has_no_loss(n, top):
    # The label's logit is one product, the others' are 0, and e^-50 is nothing beside 1: no rounding is left.
    import torch

    from paper_1612_08608_gb300 import ops
    C, d = 300, 64
    W = torch.zeros((1, C, d), device="cuda", dtype=torch.bfloat16)
    W[0, torch.arange(d), torch.arange(d)] = 1.0
    y = (torch.arange(n, device="cuda", dtype=torch.int32) * 7 % d)[None]
    X = torch.zeros((1, n, d), device="cuda", dtype=torch.bfloat16)
    X[0, torch.arange(n, device="cuda"), y[0].long()] = top
    loss, lse = ops.softmax_xent(X, W, y)
    assert bool((loss == 0).all()) and bool((lse == X.float().amax(dim=2)).all())
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, torch.ones_like(loss))
    tiny = 300 * top * 2.0 ** -72                               # e^-50 < 2^-72
    assert bool((dX.abs() <= tiny).all()) and bool((dW.abs() <= n * tiny).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,n,C,d,top", [(1, 5, 300, 32768, 10.0), (1, 5, 300, 32768, 14.0), (2, 70, 300, 16384, 10.0),
                                         (1, 20, 20000, 4096, 15.0), (3, 2, 28, 3984, 9.0)])
def test_confident_rows(N, n, C, d, top, dtype):
    # What is left of 1 of a label's probability comes from its logit as fp32 arithmetic gives it: a lane sums d / 256 groups
    # of eight products, 32 lanes join in five steps, each off by 2^-24 of the magnitudes' sum S.
    import torch

    from paper_1612_08608_gb300 import ops
    X, W, y, g = _inputs(N, n, C, d, dtype, seed=d + n, label=0.0)
    X.copy_((W[torch.arange(N, device="cuda")[:, None], y.long()].float() * top).to(X.dtype))
    loss, lse = ops.softmax_xent(X, W, y)
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g)
    _check(X, W, y, g, loss, lse, dX, dW)
    eps = torch.finfo(X.dtype).eps
    tiny = 2.0 ** -25 if X.dtype == torch.float16 else 0.0
    for i in range(N):
        x, w, at = X[i].double(), W[i].double(), torch.arange(n, device="cuda")
        z, S, yy = x @ w.T, x.abs() @ w.abs().T, y[i].long()
        p = torch.exp(z - lse[i].double()[:, None])
        hot = torch.zeros_like(p)
        hot[at, yy] = 1.0
        gg = g[i].double()[:, None]
        half = eps * eps / 4 if n <= 32 else eps / 2
        off = p * (3 * (d / 16 + 8) * 2.0 ** -23 * S.max() + half + 2.0 ** -20)
        py = p[at, yy]
        off[at, yy] = 1.5 * py * (d / 256 + 9) * 2.0 ** -24 * S[at, yy] + (half + 2.0 ** -22) * (1 - py).abs()
        off, R = gg.abs() * off, gg * (p - hot)
        small = float(gg.abs().max()) * 2.0 ** -38 if X.dtype == torch.float16 else 0.0
        for got, want, mag, err, sums in ((dX[i], R @ w, R.abs() @ w.abs(), off @ w.abs() + small * w.abs().sum(dim=0), C),
                                          (dW[i], R.T @ x, R.abs().T @ x.abs(),
                                           off.T @ x.abs() + small * x.abs().sum(dim=0), n)):
            tol = err + (sums / 16 + 16) * 2.0 ** -23 * mag + eps / 2 * want.abs() + tiny
            assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max()


@pytest.mark.parametrize("kernel,tile", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_a_wait_that_runs_out_in_short_tiles(kernel, tile):
    # as above; each of 76 clusters has two tiles or three, of twelve steps
    import torch

    from paper_1612_08608_gb300 import ops
    from paper_1612_08608_gb300._lib import load_library
    lib = load_library()
    N, n, C, d = 1, 50, 42000, 768
    X, W, y, g = _inputs(N, n, C, d, "bfloat16", seed=kernel, drop=0.1)
    _, lse = ops.softmax_xent(X, W, y)
    ws = torch.empty(max(ops.xent_workspace(N, n, C, d, grad=k)[1] for k in (False, True)), dtype=torch.uint8, device="cuda")
    assert lib.asap_debug_xent(kernel, tile, 20_000_000) == 0
    if kernel == 0:
        loss, bad = ops.softmax_xent(X, W, y, workspace=ws)
        assert bool(torch.isnan(loss[y >= 0]).all()) and bool(torch.isnan(bad[y >= 0]).all())
    else:
        dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
        assert bool(torch.isnan(dX).any()) or bool(torch.isnan(dW).any())
    assert int(ws[:4].view(torch.int32)) == 4                                  # ASAP_ERR_TIMEOUT
    loss, lse = ops.softmax_xent(X, W, y, workspace=ws)
    assert int(ws[:4].view(torch.int32)) == 0
    dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
    assert int(ws[:4].view(torch.int32)) == 0
    _check(X, W, y, g, loss, lse, dX, dW)


def test_streams_and_graphs():
    import torch

    from paper_1612_08608_gb300 import ops
    X, W, y, g = _inputs(1, 300, 2000, 192, "bfloat16", seed=6, drop=0.1)
    want = [t.clone() for t in _run(X, W, y, g)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _run(X, W, y, g)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # two graphs on one workspace, replayed in turn while the inputs (and the rows without a label) change
    ws = torch.empty(ops.xent_workspace(1, 300, 2000, 192, grad=True)[1] * 2, dtype=torch.uint8, device="cuda")
    graphs = []
    for k in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            loss, lse = ops.softmax_xent(X, W, y, workspace=ws)
            dX, dW = ops.softmax_xent_grad(X, W, y, lse, g, workspace=ws)
        graphs.append((gr, (loss, lse, dX, dW)))
    gen = torch.Generator(device="cuda").manual_seed(2)
    for turn in range(3):
        X += (0.1 * torch.randn(X.shape, generator=gen, device="cuda")).bfloat16()
        y.copy_(torch.randint(-500, 2000, y.shape, generator=gen, device="cuda"))
        ref = _run(X, W, y, g)
        for gr, out in graphs:
            gr.replay()
            _check(X, W, y, g, *out)
            assert all(torch.equal(a, b) for a, b in zip(out[:2] + out[3:], ref[:2] + ref[3:]))
