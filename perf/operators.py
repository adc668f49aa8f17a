"""Operators of per-community (per-expert) layers and of their weights' updates, as cases that can be timed.

The rows of a matrix are sorted into groups (communities of nodes, rows routed to an expert): group g owns the rows
[ptr[g], ptr[g + 1]) and has weights of its own.  A case names one operator and its sizes:

  transform     out[r] = A[r] B_g for the rows r of every group (`transposed`: B_g is stored C x K and its transpose taken,
                which is the gradient with respect to the layer's input)
  wgrad         out_g = A_g^T G_g, the gradient with respect to every group's weights, kept in 32 bits
  orthogonalise the odd polynomial X <- a X + (b S + c S^2) X, S = X X^T, applied `steps` times to every matrix of a stack over
                its Frobenius norm: its singular values go towards one
  muon          one step of an optimiser on a stack of weights: M <- mu M + G, the orthogonalised G + mu M is what is taken
                off the weights, which also decay

`run` is one pass: in plain torch operations in 32 bits where `own` is false, else the library's calls.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS, LR, MU, DECAY = 1e-7, 0.02, 0.95, 0.01


def _rows(kind, n, groups, K, C, dtype, spread, transposed=False):
    """spread: "even" groups, or "ragged" ones: log-normal shares, and every eighth group is likely to be empty."""
    return dict(kind=kind, n=n, groups=groups, K=K, C=C, dtype=dtype, spread=spread, transposed=transposed)


def _stack(kind, batch, K, C, dtype, steps=5):
    return dict(kind=kind, batch=batch, K=K, C=C, dtype=dtype, steps=steps)


def listed():
    return [
        # serving: sixteen rows on their way through sixty-four groups' weights; what counts is reading the weights that are hit
        dict(name="transform_few_rows", **_rows("transform", 16, 64, 2048, 1024, "bf16", "ragged")),
        # a hidden layer with weights per community: two hundred thousand nodes, thirty-two communities, 32 bits
        dict(name="transform_nodes", **_rows("transform", 200000, 32, 256, 256, "f32", "even")),
        # five hundred thousand nodes, a layer of 512 units, 16 bits: memory and matrix cores about alike
        dict(name="transform_wide", **_rows("transform", 500000, 16, 512, 512, "bf16", "even")),
        # experts of very different load, wide layers: bound by the matrix cores
        dict(name="transform_experts", **_rows("transform", 16384, 64, 2048, 1024, "bf16", "ragged")),
        # the input's gradient at sizes that are multiples of nothing
        dict(name="transform_odd_gradient", **_rows("transform", 30011, 7, 97, 301, "f16", "ragged", True)),
        # gradients of the weights of the three layers above
        dict(name="wgrad_nodes", **_rows("wgrad", 200000, 32, 256, 256, "f32", "even")),
        dict(name="wgrad_experts", **_rows("wgrad", 16384, 64, 2048, 1024, "bf16", "ragged")),
        # a last layer of a small graph: short sums, few columns, latency
        dict(name="wgrad_small", **_rows("wgrad", 2000, 4, 97, 7, "f32", "ragged")),
        # one small layer's update: latency
        dict(name="orthogonalise_small", **_stack("orthogonalise", 1, 256, 64, "f32")),
        # the updates of many wide layers in one stack: bound by the matrix cores
        dict(name="orthogonalise_stack", **_stack("orthogonalise", 32, 2048, 1024, "bf16")),
        # an optimiser's step on the hidden layers of an eight-layer model of 512 units
        dict(name="muon_deep", **_stack("muon", 7, 512, 512, "f32")),
        # the same on the first layer of the paper's larger graph: one ragged matrix
        dict(name="muon_ragged", **_stack("muon", 1, 767, 1000, "f32")),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["transform", "transform", "wgrad", "orthogonalise", "muon"])
    if kind in ("transform", "wgrad"):
        dtype, spread = rng.choice(["f32", "bf16", "f16"]), rng.choice(["even", "ragged"])
        K, C, groups = _log(rng, 8, 2048), _log(rng, 3, 2048), _log(rng, 1, 64)
        if rng.random() < 0.5:                                  # half of them at sizes of layers as they are mostly built
            K, C = max(K // 64, 1) * 64, max(C // 64, 1) * 64
        groups = max(1, min(groups, int(1.2e8 / (K * C))))
        most = min(300000, 1.0e11 / (2 * K * C), (2.5e8 if spread == "even" else 6e7) / (K + C))
        return _rows(kind, _log(rng, 1, max(int(most), 1)), groups, K, C, dtype, spread, kind == "transform" and rng.random() < 0.4)
    K, C = _log(rng, 16, 2048), _log(rng, 16, 2048)
    if rng.random() < 0.5:
        K, C = max(K // 64, 1) * 64, max(C // 64, 1) * 64
    most = min(64.0, 4e7 / (K * C), 4e10 / (float(K) * C * min(K, C)))
    return _stack(kind, _log(rng, 1, max(int(most), 1)), K, C, rng.choice(["f32", "bf16", "f16"]), rng.choice([5, 5, 5, 3, 6]))


def _offsets(case, seed):
    """Where the groups' rows begin: groups + 1 numbers, from 0 to n."""
    n, groups = case["n"], case["groups"]
    if case["spread"] == "even":
        return [n * g // groups for g in range(groups + 1)]
    rng = random.Random(seed)
    shares = [0.0 if rng.random() < 0.125 else math.exp(rng.gauss(0.0, 1.0)) for _ in range(groups)]
    shares[rng.randrange(groups)] += 1e-3                       # one at least
    total, ends, so_far = sum(shares), [0], 0.0
    if n < 4 * groups:                                          # few rows: each goes to a group of its own choice
        hits = rng.choices(range(groups), weights=shares, k=n)
        for g in range(groups):
            ends.append(ends[-1] + hits.count(g))
        return ends
    for s in shares:
        so_far += s
        ends.append(min(n, int(round(n * so_far / total))))
    ends[-1] = n
    return ends


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t, K, C = TYPES[case["dtype"]], case["K"], case["C"]
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    if case["kind"] in ("transform", "wgrad"):
        ends = _offsets(case, seed)
        longest = max(b - a for a, b in zip(ends, ends[1:]))
        # a layer's input is what a ReLU left; a gradient is small and has both signs
        A = randn(case["n"], K)
        A = (A * 1e-2 if case["transposed"] else A.relu_()).to(t)
        st = dict(case=case, A=A, ptr=torch.tensor(ends, dtype=torch.int64, device=DEV), longest=longest)
        if case["kind"] == "wgrad":
            st["G"] = (randn(case["n"], C) * 1e-2).to(t)
        else:
            shape = (case["groups"], C, K) if case["transposed"] else (case["groups"], K, C)
            st["B"] = ((torch.rand(shape, generator=g, device=DEV) * 2 - 1) * (6.0 / (K + C)) ** 0.5).to(t)
        return st
    # gradients of layers: a few strong directions, the others far below them
    batch, rank = case["batch"], min(16, K, C)
    strength = 0.6 ** torch.arange(rank, device=DEV)
    G = (randn(batch, K, rank) * strength) @ randn(batch, rank, C) + 0.1 * randn(batch, K, C)
    G = (G * 1e-3).to(t)
    if case["kind"] == "orthogonalise":
        return dict(case=case, G=G)
    W = (torch.rand((batch, K, C), generator=g, device=DEV) * 2 - 1) * (6.0 / (K + C)) ** 0.5
    return dict(case=case, G=G, W=W, M=randn(batch, K, C) * 1e-3)


@functools.lru_cache(maxsize=1)
def _solver():
    from paper_2112_09335_amd import binding
    return binding.Solver(0)


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        s = _solver()
        if kind == "transform":
            return s.op_transform_grouped(state["A"], state["B"], state["ptr"], transposed=case["transposed"])
        if kind == "wgrad":
            return s.op_wgrad_grouped(state["A"], state["G"], state["ptr"])
        if kind == "orthogonalise":
            return s.op_orthogonalise(state["G"], steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
        s.op_muon_step(state["W"], state["M"], state["G"], lr=LR, momentum=MU, nesterov=True, weight_decay=DECAY,
                       scale=_scale(case), steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
        return dict(W=state["W"], M=state["M"])
    if kind == "transform":
        return _transform(state["A"], state["B"], state["ptr"], state["longest"], case["transposed"])
    if kind == "wgrad":
        return _wgrad(state["A"], state["G"], state["ptr"], state["longest"])
    if kind == "orthogonalise":
        return _orthogonalise(state["G"].float(), case["steps"]).to(state["G"].dtype)
    W, M, G = state["W"], state["M"], state["G"].float()
    M.mul_(MU).add_(G)
    W.mul_(1.0 - LR * DECAY).sub_(_orthogonalise(G + MU * M, case["steps"]) * (LR * _scale(case)))
    return dict(W=W, M=M)


def _scale(case):
    return max(1.0, case["C"] / case["K"]) ** 0.5


def _places(ptr, n):
    """Group of every row and its place in it."""
    row = torch.arange(n, device=ptr.device)
    group = torch.searchsorted(ptr[1:].contiguous(), row, right=True)
    return group, row - ptr[group]


def _padded(A, group, place, groups, longest):
    out = torch.zeros((groups, longest, A.shape[1]), device=A.device)
    out[group, place] = A.float()
    return out


def _transform(A, B, ptr, longest, transposed):
    """Every group's rows padded to the longest, one batched product."""
    group, place = _places(ptr, A.shape[0])
    right = B.float().transpose(1, 2).contiguous() if transposed else B.float()
    return torch.bmm(_padded(A, group, place, B.shape[0], longest), right)[group, place].to(A.dtype)


def _wgrad(A, G, ptr, longest):
    group, place = _places(ptr, A.shape[0])
    groups = ptr.shape[0] - 1
    left = _padded(A, group, place, groups, longest).transpose(1, 2).contiguous()
    return torch.bmm(left, _padded(G, group, place, groups, longest))


def _orthogonalise(X, steps):
    a, b, c = COEFFICIENTS
    X = X / ((X * X).sum((1, 2), keepdim=True).sqrt() + EPS)
    wide = X.shape[1] <= X.shape[2]
    X = X if wide else X.transpose(1, 2).contiguous()
    for _ in range(steps):
        S = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * S + c * torch.bmm(S, S), X)
    return X if wide else X.transpose(1, 2).contiguous()


def work(case):
    """Inputs read once, results written once; of the groups' weights those that few rows can hit.  Of the symmetric products
    of the polynomial one half."""
    K, C = float(case["K"]), float(case["C"])
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}[case["dtype"]]
    if case["kind"] in ("transform", "wgrad"):
        n, groups = float(case["n"]), float(case["groups"])
        weights = size * min(n, groups) * K * C if case["kind"] == "transform" else 4.0 * groups * K * C
        return {"bytes": size * n * (K + C) + weights + 8.0 * (groups + 1), "flops": 2.0 * n * K * C}
    batch, r, s = float(case["batch"]), min(K, C), max(K, C)
    flops = batch * case["steps"] * (3.0 * r * r * s + r * r * r)
    moved = 2.0 * size if case["kind"] == "orthogonalise" else size + 16.0
    return {"bytes": moved * batch * K * C, "flops": flops}


def _exact_orthogonal(X, steps):
    """The polynomial is X times a polynomial of the smaller of X^T X and X X^T: all factors commute, so they are gathered first
    and X is multiplied once."""
    a, b, c = COEFFICIENTS
    X = X / (torch.sqrt(torch.sum(X ** 2)) + EPS)
    tall = X.shape[0] > X.shape[1]
    S = X.T @ X if tall else X @ X.T
    eye = torch.eye(S.shape[0], dtype=S.dtype, device=S.device)
    P = eye
    for _ in range(steps):
        F = a * eye + S @ (b * eye + c * S)
        P, S = P @ F, F @ S @ F
    return X @ P if tall else P @ X


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("transform", "wgrad"):
        ends = _offsets(case, seed)
        A = st["A"]
        shape = (case["n"], case["C"]) if case["kind"] == "transform" else (case["groups"], case["K"], case["C"])
        out = torch.zeros(shape, dtype=torch.float64, device=DEV)
        for g, (lo, hi) in enumerate(zip(ends, ends[1:])):
            if hi > lo and case["kind"] == "transform":
                B = st["B"][g].double()
                out[lo:hi] = A[lo:hi].double() @ (B.T if case["transposed"] else B)
            elif hi > lo:
                out[g] = A[lo:hi].double().T @ st["G"][lo:hi].double()
        return out
    G = st["G"].double()
    if case["kind"] == "orthogonalise":
        return torch.stack([_exact_orthogonal(x, case["steps"]) for x in G])
    M = MU * st["M"].double() + G
    step = torch.stack([_exact_orthogonal(x, case["steps"]) for x in MU * M + G])
    return dict(W=st["W"].double() * (1.0 - LR * DECAY) - LR * _scale(case) * step, M=M)
