"""Products grouped by expert with their gradients, and the orthogonalised update of such weights, as cases that can be timed and compared.

``listed()`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes what a program has in hand before the call,
``run`` is one pass: where ``own`` is true through the public entry points of ``paper_2112_09335_b200.binding.GcnAdmm``, else the same
operator in elementary torch operations in 32 bits.  ``exact`` gives the outputs from the definition in 64 bits.  A case is a dict of plain values:

  path     "product"     y[i] = x[i] W_g for the rows i of group g (an expert's tokens, a community's nodes)
           "gradient_x"  dx[i] = dy[i] W_g^T, the weights stored as the forward product reads them
           "gradient_w"  dW_g = sum over the rows i of group g of x[i]^T dy[i]
           "orthogonal"  steps X <- a X + (b A + c A A) X with A = X X^T, from X = G / (||G|| + eps), for every matrix of a batch
  type     of the inputs, "f32", "bf16" or "f16";  out: of the outputs
  groups, rows, k, n   number of groups; rows of x; width of x; width of y.  W_g is k x n
  skew     how unequal the groups are (deviation of the logarithm of their sizes);  empty: groups that get no row;
           tail: rows behind the last group's, which no call touches
  batch, rows, cols, steps   of "orthogonal"
"""
from __future__ import annotations

import functools
import math

import torch

own = False

TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)
SIZE = dict(f32=4, bf16=2, f16=2)
COEFFICIENTS = (3.4445, -4.7750, 2.0315)     # of a quintic step that lifts every singular value towards 1
EPS = 1e-7
SCALE = 0.2                                  # of the update


def listed():
    return [
        # The smallest call: every community of a toy graph has a first-layer weight of its own.  Launch latency is all there is.
        dict(name="product tiny", path="product", type="f32", out="f32", groups=4, rows=1000, k=128, n=16, skew=0.3, empty=0, tail=0),
        # Serving, single tokens: eight tokens in flight, each with its expert out of 64.  The experts' weights are the bytes.
        dict(name="product tokens", path="product", type="bf16", out="bf16", groups=64, rows=8, k=1024, n=2048, skew=0.5, empty=8, tail=0),
        # A padded batch in training: unequal experts, some of them idle, rows behind the last one.
        dict(name="product batch", path="product", type="bf16", out="bf16", groups=16, rows=32768, k=2048, n=2048, skew=0.4, empty=2, tail=200),
        # A weight per community on the nodes of a large graph, in the trainer's own type.
        dict(name="product communities", path="product", type="f32", out="f32", groups=32, rows=169343, k=128, n=256, skew=0.3, empty=0, tail=0),
        # Gradient of the input of the padded batch.
        dict(name="gradient_x batch", path="gradient_x", type="bf16", out="bf16", groups=16, rows=16384, k=2048, n=1024, skew=0.4, empty=2, tail=100),
        # Odd widths, which no 16-byte boundary fits, on a graph of medium size.
        dict(name="gradient_x odd", path="gradient_x", type="f16", out="f16", groups=10, rows=13752, k=767, n=1000, skew=0.4, empty=1, tail=0),
        # Gradient of the experts' weights, kept in fp32 for the optimiser.
        dict(name="gradient_w batch", path="gradient_w", type="bf16", out="f32", groups=16, rows=16384, k=2048, n=1024, skew=0.4, empty=2, tail=100),
        # Gradient of the communities' last-layer weights: few columns, long sums.
        dict(name="gradient_w communities", path="gradient_w", type="f32", out="f32", groups=32, rows=169343, k=256, n=40, skew=0.3, empty=0, tail=0),
        # Update of the small weights of a few communities.
        dict(name="orthogonal small", path="orthogonal", type="f32", out="f32", batch=8, rows=128, cols=16, steps=5),
        # Update of one weight of odd shape, taller than wide.
        dict(name="orthogonal odd", path="orthogonal", type="f32", out="f32", batch=1, rows=1000, cols=767, steps=5),
        # Update of a layer's experts.
        dict(name="orthogonal experts", path="orthogonal", type="bf16", out="bf16", batch=16, rows=1024, cols=2048, steps=5),
        # Update of one large square weight.
        dict(name="orthogonal large", path="orthogonal", type="bf16", out="bf16", batch=1, rows=4096, cols=4096, steps=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    path = rng.choice(["product", "product", "gradient_x", "gradient_w", "gradient_w", "orthogonal"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if path == "orthogonal":
        batch = _log_int(rng, 1, 32)
        return dict(path=path, type=kind, out=kind, batch=batch, rows=_log_int(rng, 7, 2500), cols=_log_int(rng, 7, 2500), steps=rng.randint(3, 6))
    groups = _log_int(rng, 1, 128)
    even = rng.random() < 0.6                     # widths of a model (multiples of 8), or any
    def width():
        w = _log_int(rng, 7, 2500)
        return max(8, w // 8 * 8) if even else w
    k, n = width(), width()
    return dict(path=path, type=kind, out="f32" if kind != "f32" and rng.random() < 0.4 else kind, groups=groups, rows=_log_int(rng, 1, 200000), k=k, n=n,
                skew=round(rng.uniform(0.0, 0.6), 2), empty=rng.randint(0, groups // 4), tail=rng.choice([0, 0, 1, 77]))


def draw(rng):
    """One more case of the ranges of ``listed`` that costs at most half of the dearest listed product."""
    while True:
        case = _draw_once(rng)
        w = work(case)
        if w["bytes"] <= 1e9 and w["flops"] <= (1.5e11 if case["path"] != "orthogonal" else 5e11):
            return case


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once, and the multiplications of the formulas."""
    a, b = SIZE[case["type"]], SIZE[case["out"]]
    if case["path"] == "orthogonal":
        m, n = sorted((case["rows"], case["cols"]))
        # A, A A are symmetric: one triangle has to be formed
        flops = case["steps"] * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)
        return dict(bytes=float(case["batch"] * m * n * (a + b)), flops=float(case["batch"] * flops))
    k, n, rows = case["k"], case["n"], case["rows"]
    flops = 2.0 * rows * k * n
    if case["path"] == "gradient_w":
        return dict(bytes=float(rows * (k + n) * a + case["groups"] * k * n * b), flops=flops)
    full = case["groups"] - case["empty"]
    met = full * (1.0 - (1.0 - 1.0 / full) ** rows)              # groups that hold a row
    return dict(bytes=rows * ((k if case["path"] == "product" else n) * a + (n if case["path"] == "product" else k) * b) + met * k * n * a, flops=flops)


# ---- inputs ----------------------------------------------------------------------------------------

def _counts(case, gen):
    """Rows of every group: whole numbers that add up to case["rows"], a few groups without any."""
    groups, rows = case["groups"], case["rows"]
    share = torch.exp(case["skew"] * torch.randn(groups, generator=gen, dtype=torch.float64))
    share[torch.randperm(groups, generator=gen)[:case["empty"]]] = 0.0
    if rows <= 4 * groups:
        return torch.bincount(torch.multinomial(share, rows, replacement=True, generator=gen), minlength=groups)
    count = (share / share.sum() * rows).to(torch.int64)
    count[torch.argmax(share)] += rows - int(count.sum())
    return count


def prepare(case, seed):
    """Inputs, and where ``own`` is true the handle of the current device and stream: passes are enqueued on the stream that was current here."""
    state = _inputs(case, seed)
    if own:
        state["handle"] = _trainer(torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)
    return state


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)
    kind, out = TYPES[case["type"]], TYPES[case["out"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(kind)
    if case["path"] == "orthogonal":
        b, m, n = case["batch"], case["rows"], case["cols"]
        # a gradient: a few strong directions above a floor of noise
        strong = torch.randn(b, m, 4, generator=gen, device="cuda") @ torch.randn(b, 4, n, generator=gen, device="cuda")
        g = ((strong + torch.randn(b, m, n, generator=gen, device="cuda")) * 1e-3).to(kind)
        return dict(case=case, g=g, out=torch.empty(b, m, n, dtype=out, device="cuda"))
    count = _counts(case, torch.Generator().manual_seed(1000003 * seed + 29))
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(count, 0)])
    k, n, groups, held = case["k"], case["n"], case["groups"], case["rows"] + case["tail"]
    state = dict(case=case, held=held, offsets=offsets.to(torch.int32).cuda(), largest=max(1, int(count.max())))
    if case["path"] == "gradient_w":
        state["x"], state["dy"] = normal(held, k), normal(held, n, scale=1e-2)
        state["out"] = torch.empty(groups, k, n, dtype=out, device="cuda")
        return state
    w = torch.empty(groups, k, n, dtype=kind, device="cuda")
    for g in range(groups):                       # a group at a time: no fp32 copy of all weights
        w[g] = normal(k, n, scale=k ** -0.5)
    state["w"] = w
    if case["path"] == "product":
        state["x"] = normal(held, k)
        state["out"] = torch.zeros(held, n, dtype=out, device="cuda")
    else:
        state["dy"] = normal(held, n, scale=1e-2)
        state["out"] = torch.zeros(held, k, dtype=out, device="cuda")
    return state


# ---- one pass --------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _trainer(device, stream):
    """The handle that a program keeps for a device and a stream: its workspace serves the calls."""
    import numpy as np

    from paper_2112_09335_b200 import binding
    one = np.ones((2, 1), dtype=np.float32)
    return binding.GcnAdmm(2, np.array([0, 1, 2]), np.array([1, 0]), one, np.zeros(2), np.ones(2), [1, 1], 1, np.zeros(2), [one[:1]], stream=stream,
                           device=device)


def _own(state):
    from paper_2112_09335_b200 import binding
    case, out, h = state["case"], state["out"], state["handle"]
    types = dict(type=getattr(binding, case["type"].upper()), out_type=getattr(binding, case["out"].upper()))
    if case["path"] == "orthogonal":
        h.orthogonalise(state["g"].data_ptr(), out.data_ptr(), case["batch"], case["rows"], case["cols"], coefficients=[COEFFICIENTS] * case["steps"],
                        eps=EPS, scale=SCALE, **types)
        return out
    offsets, groups, rows, k, n = state["offsets"].data_ptr(), case["groups"], state["held"], case["k"], case["n"]
    if case["path"] == "product":
        h.grouped_product(state["x"].data_ptr(), state["w"].data_ptr(), out.data_ptr(), offsets, groups, rows, k, n, **types)
    elif case["path"] == "gradient_x":
        h.grouped_product(state["dy"].data_ptr(), state["w"].data_ptr(), out.data_ptr(), offsets, groups, rows, n, k, transpose_w=True, **types)
    else:
        h.grouped_product_tn(state["x"].data_ptr(), state["dy"].data_ptr(), out.data_ptr(), offsets, groups, rows, k, n, **types)
    return out


def _padded(x, at, inside):
    """x's rows by group, groups x largest x width in fp32, zero where a group has fewer."""
    return torch.where(inside[..., None], x[at].float(), 0.0)


def _plain_orthogonal(state):
    case = state["case"]
    x = state["g"].float()
    x = x.mT if case["rows"] > case["cols"] else x
    x = (x.double() / (x.double().square().sum((1, 2), keepdim=True).sqrt() + EPS)).float()
    a, b, c = COEFFICIENTS
    for _ in range(case["steps"]):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    x = SCALE * x
    state["out"].copy_(x.mT if case["rows"] > case["cols"] else x)
    return state["out"]


def run(state):
    if own:
        return _own(state)
    case, out = state["case"], state["out"]
    if case["path"] == "orthogonal":
        return _plain_orthogonal(state)
    offsets = state["offsets"].long()
    if case["path"] != "gradient_w" and case["rows"] <= case["groups"]:      # fewer rows than groups: each row with its own weights
        x = state["x" if case["path"] == "product" else "dy"][:case["rows"]]
        at = torch.arange(case["rows"], device="cuda")
        w = state["w"][torch.searchsorted(offsets, at, right=True) - 1].float()
        out[:case["rows"]] = (x.float()[:, None] @ (w if case["path"] == "product" else w.mT))[:, 0].to(out.dtype)
        return out
    at = offsets[:-1, None] + torch.arange(state["largest"], device="cuda")
    inside = at < offsets[1:, None]
    at = at.clamp(max=state["held"] - 1)
    if case["path"] == "gradient_w":
        out.copy_(_padded(state["x"], at, inside).mT @ _padded(state["dy"], at, inside))
        return out
    w = state["w"].float()
    y = _padded(state["x"] if case["path"] == "product" else state["dy"], at, inside) @ (w if case["path"] == "product" else w.mT)
    out[at[inside]] = y[inside].to(out.dtype)
    return out


# ---- the definition in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    state = _inputs(case, seed)
    if case["path"] == "orthogonal":
        a, b, c = COEFFICIENTS
        made = []
        for g in state["g"]:
            x = g.double() if case["rows"] <= case["cols"] else g.double().T
            x = x / (torch.linalg.norm(x) + EPS)
            # every step multiplies X by a polynomial of X X^T, and these commute: the factors are gathered in Q, the last product is with X
            one = torch.eye(len(x), dtype=torch.float64, device="cuda")
            s, q = x @ x.T, one
            for _ in range(case["steps"]):
                p = a * one + b * s + c * (s @ s)
                q, s = p @ q, p @ s @ p
            x = SCALE * (q @ x)
            made.append(x if case["rows"] <= case["cols"] else x.T)
        return torch.stack(made)
    offsets = state["offsets"].tolist()
    out = torch.zeros(state["out"].shape, dtype=torch.float64, device="cuda")
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if case["path"] == "product":
            out[lo:hi] = state["x"][lo:hi].double() @ state["w"][g].double()
        elif case["path"] == "gradient_x":
            out[lo:hi] = state["dy"][lo:hi].double() @ state["w"][g].double().T
        else:
            out[g] = state["x"][lo:hi].double().T @ state["dy"][lo:hi].double()
    return out
