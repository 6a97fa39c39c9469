"""Cases that measure the context-free operators of training a large-vocabulary head data-parallel:

  loss   softmax cross entropy of z = x . w over a vocabulary, forward only (evaluation, scoring);
  train  the same and its gradients with respect to the features and the head, as a training step calls them;
  clip   the global gradient norm of each worker's tensors, and the gradients scaled to a largest norm;
  sgd    the SGD step with clipped gradients on fp32 parameters that keep a 16-bit copy.

N workers have a head and features each (N = 1: an ordinary model).  Labels below 0 leave a row out.  ``run``
in its plain form is elementary torch in 32 bits; ``exact`` restates the definitions in 64 bits."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LARGEST = 4096 * 131072 * 4096     # rows x vocabulary x features, all workers: no case is larger


def listed():
    return [
        # The next token of one sequence is scored: one row against a whole head.  Latency and the head's bytes.
        dict(name="loss one token", kind="loss", N=1, n=1, C=32000, d=2048, dtype="bf16", ignore=0.0, ld=0),
        # Perplexity of a batch of documents, prompts left out, on an odd vocabulary in fp16.
        dict(name="loss eval documents", kind="loss", N=1, n=4095, C=50001, d=2048, dtype="fp16", ignore=0.3, ld=0),
        # The smallest dense configuration of the tests: four workers, ten classes.
        dict(name="train small workers", kind="train", N=4, n=128, C=10, d=256, dtype="bf16", ignore=0.0, ld=0),
        # The benchmark's dense configuration.
        dict(name="train bench workers", kind="train", N=32, n=512, C=1000, d=2048, dtype="bf16", ignore=0.0, ld=0),
        # Few rows against a large head: the head's bytes are what counts.
        dict(name="train few rows", kind="train", N=1, n=64, C=131072, d=2048, dtype="bf16", ignore=0.0, ld=0),
        # Fine-tuning on answers: more than half of the labels are prompts and padding; odd sizes, padded rows, fp16.
        dict(name="train answers only", kind="train", N=1, n=4099, C=49999, d=1999, dtype="fp16", ignore=0.6, ld=2048),
        # Pre-training: a whole batch against a large head.
        dict(name="train large", kind="train", N=1, n=4096, C=131072, d=4096, dtype="bf16", ignore=0.0, ld=0),
        # The gradients of a small model: latency.
        dict(name="clip small model", kind="clip", tensors=6, elements=20000, groups=1, dtype="fp32", packed=False, shapes=1),
        # Every one of the benchmark's dense workers clips its own gradient.
        dict(name="clip workers", kind="clip", tensors=32, elements=32 * 2048000, groups=32, dtype="bf16", packed=False, shapes=0),
        # A whole model: many tensors of very different sizes, packed one behind the other, larger than L2.
        dict(name="clip whole model", kind="clip", tensors=290, elements=1 << 30, groups=1, dtype="bf16", packed=True, shapes=2),
        # The step of a small head on each of eight workers.
        dict(name="sgd workers", kind="sgd", tensors=16, elements=8 * 300000, groups=8, dtype="fp32", packed=False, shapes=3),
        # The step of a whole model with bf16 gradients.
        dict(name="sgd whole model", kind="sgd", tensors=180, elements=1 << 29, groups=1, dtype="bf16", packed=True, shapes=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["loss", "train", "train", "clip", "sgd"])
    if kind in ("loss", "train"):
        N = rng.choice([1, 1, 1, 2, 4, 8, 16, 32])
        d = 8 * _log(rng, 2, 512) if rng.random() < 0.75 else _log(rng, 16, 4096)
        C = _log(rng, 10, min(131072, (1 << 29) // (N * d)))
        n = _log(rng, 1, min(8192, (1 << 25) // (N * d), LARGEST // (N * C * d)))
        ld = (d + 7) // 8 * 8 + 64 if rng.random() < 0.25 else 0
        return dict(kind=kind, N=N, n=n, C=C, d=d, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                    ignore=rng.choice([0.0, 0.0, 0.2, 0.5, 0.9]), ld=ld)
    tensors = _log(rng, 1, 400)
    return dict(kind=kind, tensors=tensors, elements=_log(rng, max(1000, 4 * tensors), 1 << (30 if kind == "clip" else 29)),
                groups=rng.choice([1, 1, min(tensors, 4), min(tensors, 32)]), dtype=rng.choice(["fp32", "bf16", "fp16"]),
                packed=rng.random() < 0.5, shapes=rng.randrange(1000))


# ---- inputs ---------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + salt)
    return g


def _rows(shape, ld, gen, dtype, scale):
    """[N, rows, d] in rows of ld elements (0: as many as a multiple of 16 bytes takes)."""
    N, rows, d = shape
    ld = ld or (d + 7) // 8 * 8
    x = torch.zeros((N, rows, ld), device="cuda", dtype=dtype)
    for i in range(N):                        # a worker at a time, so that little is held in 32 bits
        x[i, :, :d] = (torch.randn((rows, d), generator=gen, device="cuda") * scale).to(dtype)
    return x[:, :, :d]


def _sizes(case):
    """Elements of every tensor: a few large matrices and many small ones, of odd sizes among them."""
    T, total, G = case["tensors"], case["elements"], case["groups"]
    if case["shapes"] == 0 or T == 1:
        return [total // T] * T
    r = random.Random(case["shapes"])
    each = [math.exp(r.uniform(0.0, 7.0)) for _ in range(T)]
    return [max(1, int(total * e / sum(each))) for e in each]


def _bucket(sizes, dtype, packed):
    """Views of one flat buffer, at odd offsets if packed, else 256 bytes aligned."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += n if packed else (n + 127) // 128 * 128
    flat = torch.zeros(at, device="cuda", dtype=dtype)
    return flat, [flat[p:p + n] for p, n in zip(places, sizes)]


def prepare(case, seed):
    s = dict(case)
    dtype = DTYPES[case["dtype"]]
    if case["kind"] in ("loss", "train"):
        N, n, C, d = case["N"], case["n"], case["C"], case["d"]
        s["W"] = _rows((N, C, d), case["ld"], _gen(seed, 1), dtype, 1.0 / math.sqrt(d))
        s["X"] = _rows((N, n, d), case["ld"], _gen(seed, 2), dtype, 1.0)
        y = torch.randint(0, C, (N, n), generator=_gen(seed, 3), device="cuda")
        # a model in training: the label's logit is raised, by less for some rows than for others
        up = 12.0 * torch.rand((N, n, 1), generator=_gen(seed, 4), device="cuda")
        pick = torch.arange(N, device="cuda").unsqueeze(1)
        s["X"].add_((up * s["W"][pick, y].float()).to(dtype))
        # prompts and padding: runs of rows without a label
        run_of = torch.rand((N, n // 37 + 1), generator=_gen(seed, 5), device="cuda")
        run_of[:, 0] = 1.0                                       # some rows always have one
        run_of = run_of.repeat_interleave(37, dim=1)[:, :n]
        y = torch.where(run_of < case["ignore"], torch.full_like(y, -100), y)
        s["y"] = y.to(torch.int32)
        # the mean over a worker's rows with a label; fp16 runs scale their loss
        count = (y >= 0).sum(dim=1, keepdim=True).clamp(min=1)
        up16 = 1024.0 if dtype == torch.float16 else 1.0
        s["g"] = (up16 / count).expand(N, n).float().contiguous()
        return s
    sizes = _sizes(case)
    flat, s["grads"] = _bucket(sizes, dtype, case["packed"])
    gen = _gen(seed, 6)
    for k, v in enumerate(s["grads"]):        # tensors of a model have gradients of different sizes
        v.copy_(torch.randn(v.numel(), generator=gen, device="cuda") * 10.0 ** (k % 3 - 3))
    s["group_of"] = [k * case["groups"] // case["tensors"] for k in range(case["tensors"])]
    if case["kind"] == "clip":
        s["flat"], s["out"] = _bucket(sizes, dtype, case["packed"])
    else:
        s["flat"], s["params"] = _bucket(sizes, torch.float32, case["packed"])
        s["flat"].normal_(generator=gen)
        s["flat16"], s["copies"] = _bucket(sizes, torch.bfloat16, case["packed"])
    # norms lie around the largest one: some groups are clipped and some are not
    s["max_norm"] = 0.7 * math.sqrt(sum(float(n) * 100.0 ** (k % 3 - 3) for k, n in enumerate(sizes)) / case["groups"])
    s["lr"], s["l2"] = 0.01, 1e-4
    return s


# ---- one pass ---------------------------------------------------------------------------------------------
def _loss(X, W, y):
    z = X @ W.mT
    top = z.max(dim=2, keepdim=True).values
    lse = torch.log(torch.exp(z - top).sum(dim=2)) + top.squeeze(2)
    seen = y >= 0
    at = torch.where(seen, y, 0).long().unsqueeze(2)
    loss = lse - torch.gather(z, 2, at).squeeze(2)
    return z, seen, at, torch.where(seen, loss, 0.0), torch.where(seen, lse, 0.0)


def _train(X, W, y, g):
    z, seen, at, loss, lse = _loss(X, W, y)
    p = torch.exp_(z.sub_(lse.unsqueeze(2)))
    p.scatter_add_(2, at, torch.full_like(at, -1, dtype=p.dtype))
    p = torch.where(seen.unsqueeze(2), p * g.unsqueeze(2), 0.0)
    return loss, lse, p @ W, p.mT @ X


def _norms(grads, group_of, groups):
    each = torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads])
    of = torch.tensor(group_of, device=each.device)
    return torch.zeros(groups, dtype=torch.float64, device=each.device).index_add_(0, of, each).sqrt().float()


def run(s):
    kind = s["kind"]
    if own:
        from paper_1612_08608_gb300 import ops
        if kind == "loss":
            return ops.softmax_xent(s["X"], s["W"], s["y"])
        if kind == "train":
            loss, lse = ops.softmax_xent(s["X"], s["W"], s["y"])
            dX, dW = ops.softmax_xent_grad(s["X"], s["W"], s["y"], lse, s["g"])
            return loss, lse, dX, dW
        if kind == "clip":
            norms = ops.clip_grads(s["grads"], s["max_norm"], out=s["out"], groups=s["group_of"])
            return s["flat"], norms
        if "begun" not in s:          # the copies start as the parameters, as a program makes them once
            s["begun"] = s["flat16"].copy_(s["flat"])
        norms = ops.sgd_step(s["params"], s["grads"], s["lr"], s["max_norm"], l2=s["l2"], copies=s["copies"],
                             groups=s["group_of"])
        return s["flat"], s["flat16"], norms
    if kind == "loss":
        return _loss(s["X"].float(), s["W"].float(), s["y"])[3:]
    if kind == "train":
        dtype = s["X"].dtype
        loss, lse, dX, dW = _train(s["X"].float(), s["W"].float(), s["y"], s["g"])
        return loss, lse, dX.to(dtype), dW.to(dtype)
    norms = _norms(s["grads"], s["group_of"], s["groups"])
    scale = torch.where(norms > s["max_norm"], s["max_norm"] / norms, 1.0)
    if kind == "clip":
        [o.copy_(g.float() * scale[k]) for o, g, k in zip(s["out"], s["grads"], s["group_of"])]
        return s["flat"], norms
    [w.mul_(1.0 - s["lr"] * s["l2"]).sub_((s["lr"] * scale[k]) * g.float())
     for w, g, k in zip(s["params"], s["grads"], s["group_of"])]
    s["flat16"].copy_(s["flat"])
    return s["flat"], s["flat16"], norms


# ---- what a pass cannot do without ------------------------------------------------------------------------
def work(case):
    if case["kind"] in ("loss", "train"):
        N, n, C, d = case["N"], case["n"], case["C"], case["d"]
        n = max(1.0, n * (1.0 - case["ignore"]))                # rows without a label need no work
        if case["kind"] == "loss":
            return dict(bytes=N * (2.0 * (n + C) * d + 12.0 * n), flops=2.0 * N * n * C * d)
        # loss: X, W; gradients: X, W again; dX, dW; the logits twice, for they are not kept, and two products
        return dict(bytes=N * (6.0 * (n + C) * d + 24.0 * n), flops=8.0 * N * n * C * d)
    E, size = float(sum(_sizes(case))), 4.0 if case["dtype"] == "fp32" else 2.0
    if case["kind"] == "clip":
        return dict(bytes=2.0 * size * E, flops=3.0 * E)
    return dict(bytes=(size + 10.0) * E, flops=6.0 * E)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("loss", "train"):
        N, n, C, d = case["N"], case["n"], case["C"], case["d"]
        if N * n * C * d * (6 if case["kind"] == "train" else 2) > 1.4e13:
            return None                                          # over about 20 s in 64 bits
        loss = torch.zeros((N, n), dtype=torch.float64, device="cuda")
        lse = torch.zeros_like(loss)
        dX = torch.zeros((N, n, d), dtype=torch.float64, device="cuda")
        dW = torch.zeros((N, C, d), dtype=torch.float64, device="cuda")
        for i in range(N):
            rows = torch.nonzero(s["y"][i] >= 0).flatten()
            W = s["W"][i].double()
            for part in rows.split(2048):
                x, y = s["X"][i, part].double(), s["y"][i, part].long()
                logp = torch.nn.functional.log_softmax(x @ W.T, dim=1)
                own_logit = (x * W[y]).sum(dim=1)
                loss[i, part] = -logp[torch.arange(len(part), device="cuda"), y]
                lse[i, part] = loss[i, part] + own_logit
                if case["kind"] == "train":
                    r = logp.exp_()
                    r[torch.arange(len(part), device="cuda"), y] -= 1.0
                    r *= s["g"][i, part].double().unsqueeze(1)
                    dX[i, part] = r @ W
                    dW[i] += r.T @ x
        return (loss, lse) if case["kind"] == "loss" else (loss, lse, dX, dW)
    squares = [0.0] * case["groups"]
    for v, k in zip(s["grads"], s["group_of"]):
        squares[k] += float(v.double().pow(2).sum())
    norms = [math.sqrt(v) for v in squares]
    scale = [s["max_norm"] / v if v > s["max_norm"] else 1.0 for v in norms]
    flat = s["flat"].double()
    at = [v.storage_offset() for v in (s["out"] if case["kind"] == "clip" else s["params"])]
    for v, k, p in zip(s["grads"], s["group_of"], at):
        here = flat[p:p + v.numel()]
        if case["kind"] == "clip":
            here.copy_(v.double() * scale[k])
        else:
            here.mul_(1.0 - s["lr"] * s["l2"]).sub_(v.double(), alpha=s["lr"] * scale[k])
    norms = torch.tensor(norms, dtype=torch.float64)
    return (flat, norms) if case["kind"] == "clip" else (flat, flat.clone(), norms)
