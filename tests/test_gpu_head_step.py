"""The context-free operators together, as a data-parallel step of a large-vocabulary head uses them (GPU): every worker's
loss and gradient, its clipped SGD step on an fp32 head with a bf16 copy, then the stochastic reduce of the heads
(asap_mix_noalloc), several rounds, eagerly and as one captured graph, against a restatement in 64 bits.

The restatement starts each round from the GPU's own parameters and copies, so that a round's tolerances do not add up:
dW is off by at most 2 x 2^-8 of the magnitudes it sums (the roundings of R and of the result), which lr scale takes into
the heads; the reduce adds k + 1 roundings of fp32."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

N, n, V, d, lr, l2, max_norm = 4, 150, 1300, 104, 0.5, 0.01, 0.4


def _round(lib, ops, s):
    import torch
    loss, lse = ops.softmax_xent(s["X"], s["copy"], s["y"])
    s["loss"].copy_(loss)
    _, dW = ops.softmax_xent_grad(s["X"], s["copy"], s["y"], lse, s["g"], need_dX=False, dW=s["dW"])
    ops.sgd_step(list(s["W"]), list(dW), lr, max_norm, l2=l2, groups=list(range(N)), norms=s["norms"])
    p = C.c_void_p
    st = lib.asap_mix_noalloc(p(s["W"].data_ptr()), p(s["mixed"].data_ptr()), N, V * d, V * d, p(s["nbr"].data_ptr()),
                              p(s["wgt"].data_ptr()), 2, p(s["cons"].data_ptr()), p(torch.cuda.current_stream().cuda_stream))
    assert st == 0, lib.asap_last_error(None)
    s["W"].copy_(s["mixed"])
    s["copy"].copy_(s["mixed"])


def _state(seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *shape: torch.randn(shape, generator=gen, device="cuda")      # noqa: E731
    W = f(N, V, d) * d ** -0.5
    y = torch.randint(0, V, (N, n), generator=gen, device="cuda").to(torch.int32)
    y[1, 40:100] = -1
    nbr = torch.tensor([[i, (i + 1) % N] for i in range(N)], dtype=torch.int32, device="cuda")
    count = (y >= 0).sum(dim=1, keepdim=True).float()
    return dict(X=f(N, n, d).bfloat16(), W=W, copy=W.bfloat16(), y=y, g=(1.0 / count).expand(N, n).contiguous(),
                dW=torch.empty(N, V, d, dtype=torch.bfloat16, device="cuda"), mixed=torch.empty_like(W),
                norms=torch.empty(N, device="cuda"), loss=torch.empty(N, n, device="cuda"), nbr=nbr,
                wgt=torch.full((N, 2), 0.5, device="cuda"), cons=torch.empty(1, device="cuda"))


def _check(before, s):
    """One round from `before` = (W, copy)."""
    import torch
    W0, c0 = before[0].double(), before[1].double()
    half, tol = torch.empty_like(W0), torch.empty_like(W0)
    for i in range(N):
        rows = torch.nonzero(s["y"][i] >= 0).flatten()
        x, yy = s["X"][i][rows].double(), s["y"][i][rows].long()
        z = x @ c0[i].T
        lse = torch.logsumexp(z, 1)
        loss = lse - z[torch.arange(len(rows)), yy]
        assert bool(((s["loss"][i][rows] - loss).abs() <= 1e-5).all())       # 104 products a logit, of a few units
        r = torch.exp(z - lse[:, None])
        a = r.clone()
        r[torch.arange(len(rows)), yy] -= 1.0
        a[torch.arange(len(rows)), yy] += 1.0
        grad, mag = r.T @ x / len(rows), a.T @ x.abs() / len(rows)
        err = 2 * 2.0 ** -8 * mag
        norm = float(grad.norm())
        scale = max_norm / norm if norm > max_norm else 1.0
        # the norm moves by at most the norm of the errors
        assert abs(s["norms"][i].item() - norm) <= float(err.norm())
        half[i] = (1 - lr * l2) * W0[i] - lr * scale * grad
        tol[i] = lr * scale * (err + grad.abs() * float(err.norm()) / norm) + 2.0 ** -21 * W0[i].abs()
    nxt = [(i + 1) % N for i in range(N)]
    want, tol = 0.5 * (half + half[nxt]), 0.5 * (tol + tol[nxt]) + 2.0 ** -22 * half.abs()
    assert bool(((s["W"] - want).abs() <= tol).all()), ((s["W"] - want).abs() / tol).max()
    assert torch.equal(s["copy"], s["W"].bfloat16())


def test_rounds_of_loss_gradient_step_and_reduce():
    import torch

    from paper_1612_08608_gb300 import ops
    from paper_1612_08608_gb300._lib import load_library
    lib = load_library()
    s = _state(0)
    for _ in range(3):
        before = s["W"].clone(), s["copy"].clone()
        _round(lib, ops, s)
        _check(before, s)
    # the same rounds as one captured graph
    t = _state(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _round(lib, ops, t)
    t["W"].copy_(_state(0)["W"])
    t["copy"].copy_(t["W"])
    for _ in range(3):
        graph.replay()
    assert np.array_equal(t["W"].cpu().numpy(), s["W"].cpu().numpy())


def test_a_worker_whose_gradient_is_not_finite_takes_no_step():
    import torch

    from paper_1612_08608_gb300 import ops
    from paper_1612_08608_gb300._lib import load_library
    s = _state(1)
    s["X"][2, 0, 0] = float("inf")
    before = s["W"].clone()
    loss, lse = ops.softmax_xent(s["X"], s["copy"], s["y"])
    _, dW = ops.softmax_xent_grad(s["X"], s["copy"], s["y"], lse, s["g"], need_dX=False)
    norms = ops.sgd_step(list(s["W"]), list(dW), lr, max_norm, groups=list(range(N)))
    moved = [not torch.equal(s["W"][i], before[i]) for i in range(N)]
    assert moved == [True, True, False, True] and not bool(torch.isfinite(norms[2]))
    assert load_library().asap_last_error(None) is not None
