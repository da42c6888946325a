"""Training operators of the library as its users call them, in plain form and through the library, for timing and for
comparing outputs.

Between the features and the gradient of the kernels a training program normalises the feature rows, and between that
gradient and its optimiser it clips.  The operators are

  layer_norm           rocket_layer_norm: rows of features (or of any model's activations), with or without statistics
  layer_norm_backward  rocket_layer_norm_backward: gradients of the rows, the gain and the bias
  grad_norm            rocket_grad_norm: the 2-norm over all tensors of a model's gradient
  clip_grad_norm       rocket_clip_grad_norm: the norm, and the gradients scaled down to a largest norm

Sizes: rows of 20,000 pooled features (10,000 kernels), 9,996 MINIROCKET features, minibatches of 32 and the regressor's
677 training examples; the gradients of 1,000 and 10,000 kernels with those of a norm and a linear head; and generic ones
for wider models: token rows, short odd rows, stacks of square and four-fold matrices in one packed bucket.
"""
import math
import random

import torch

own = False

EPS = 1e-5
MAX_NORM = 1.0
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # one example off the production line, normalised before a trained head: latency
        dict(name="norm one example", op="layer_norm", N=1, P=20000, x="f32", y="f32", w="f32", pad=0, stats=False),
        # the forward pass of a training minibatch at paper scale, statistics kept for the backward pass
        dict(name="norm minibatch", op="layer_norm", N=32, P=20000, x="f32", y="f32", w="f32", pad=0, stats=True),
        # the whole training set's features, handed on in half the bytes to a matrix product
        dict(name="norm training set", op="layer_norm", N=677, P=20000, x="f32", y="bf16", w="f32", pad=0, stats=True),
        # activations of a wide model: many rows of a power of two
        dict(name="norm token rows", op="layer_norm", N=16384, P=4096, x="bf16", y="bf16", w="bf16", pad=0, stats=True),
        # very many short rows of odd length, no row but the first on a 16-byte border
        dict(name="norm short odd rows", op="layer_norm", N=100003, P=257, x="f16", y="f16", w="f32", pad=0, stats=False),
        # the backward pass of the minibatch: dx is what the soft transform's backward pass takes
        dict(name="norm backward minibatch", op="layer_norm_backward", N=32, P=20000, x="f32", y="f32", w="f32", pad=0),
        # MINIROCKET features of the training set in a wider buffer, gradients of a half-precision head
        dict(name="norm backward training set", op="layer_norm_backward", N=677, P=9996, x="f32", y="bf16", w="f32", pad=4),
        # the wide model's rows again
        dict(name="norm backward token rows", op="layer_norm_backward", N=16384, P=4096, x="bf16", y="bf16", w="bf16", pad=0),
        # the gradient of a small problem's kernels and head: the smallest call
        dict(name="gradient norm kernels", op="grad_norm", kind="kernels", K=1000, C=3, g="f32", scale=3.0),
        # a stack of layers, half-precision gradients in one bucket: many tensors, the largest call
        dict(name="gradient norm layers", op="grad_norm", kind="layers", depth=24, width=1024, g="bf16", scale=2.0),
        # the gradient of the paper's 10,000 kernels on 20 channels, clipped
        dict(name="clip kernels", op="clip_grad_norm", kind="kernels", K=10000, C=20, g="f32", to="f32", scale=4.0),
        # layers of odd width: no matrix on a 16-byte border, half-precision gradients to single-precision ones
        dict(name="clip odd layers", op="clip_grad_norm", kind="layers", depth=6, width=769, g="f16", to="f32", scale=5.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


#: A drawn case moves no more bytes than the largest listed one of its kind.
_MOST_BYTES = {"layer_norm": 2.7e8, "layer_norm_backward": 4.0e8, "grad_norm": 6.0e8, "clip_grad_norm": 2.6e8}


def draw(rng):
    """One more case of the same ranges: one row to 100,000, rows of 4 to 60,000 values, packed or in wider buffers;
    gradients of 50 to 20,000 kernels, or of 1 to 24 layers of width 16 to 1,100."""
    op = rng.choice(["layer_norm", "layer_norm", "layer_norm_backward", "layer_norm_backward", "grad_norm", "clip_grad_norm"])
    while True:
        if op.startswith("layer_norm"):
            x, y = rng.choice([("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
            case = dict(op=op, N=_log_int(rng, 1, 100000), P=_log_int(rng, 4, 60000), x=x, y=y, w=rng.choice(["f32", y]),
                        pad=rng.choice([0, 0, 0, 1, 8, 40]))
            if op == "layer_norm":
                case["stats"] = rng.random() < 0.6
        else:
            kind = rng.choice(["kernels", "layers"])
            g = "f32" if kind == "kernels" else rng.choice(["f32", "bf16", "f16"])
            case = dict(op=op, kind=kind, g=g, scale=round(math.exp(rng.uniform(math.log(0.2), math.log(20.0))), 3))
            if kind == "kernels":
                case.update(K=_log_int(rng, 50, 20000), C=rng.choice([1, 2, 3, 6, 9, 12, 20, 20, 32]))
            else:
                case.update(depth=_log_int(rng, 1, 24), width=_log_int(rng, 16, 1100))
            if op == "clip_grad_norm":
                case["to"] = rng.choice([g, "f32"])
        if work(case)["bytes"] <= _MOST_BYTES[op]:
            return case


def _sizes(case):
    """Lengths of the gradient tensors of a model, by the case alone."""
    if case["kind"] == "kernels":
        # weights of kernels of 7, 9 or 11 taps on some of the channels, biases, gain and bias of the norm, linear head
        rng, K = random.Random(8527), case["K"]
        weights = 0
        for _ in range(K):
            taps = rng.choice([7, 9, 11])
            weights += taps * int(2 ** rng.uniform(0, math.log2(min(case["C"], taps) + 1)))
        return [weights, K, 2 * K, 2 * K, 2 * K, 1]
    w = case["width"]
    # four square matrices, two four-fold ones, their biases, gain and bias of two norms
    layer = [w * w, w, w * w, w, w * w, w, w * w, w, 4 * w * w, 4 * w, 4 * w * w, w, w, w, w, w]
    return layer * case["depth"]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _rows(N, P, pad, dtype):
    """[N, P], the rows `pad` values apart."""
    return torch.empty((N, P + pad), dtype=dtype, device="cuda")[:, :P]


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    state = {"op": op}
    if op.startswith("layer_norm"):
        N, P, pad = case["N"], case["P"], case["pad"]
        x = torch.randn((N, P), generator=gen, device="cuda")
        if case["x"] == "f32":
            # pooled features: shares of positive outputs in [0, 1] and maxima of order 1, in turn
            x[:, 0::2] = torch.special.ndtr(x[:, 0::2])
            x[:, 1::2] = 2.0 + 0.7 * x[:, 1::2]
        else:
            # activations: unit scale, a few channels far above it
            scale = torch.where(torch.rand((P,), generator=gen, device="cuda") < 0.01, 12.0, 1.0)
            x = x * scale + 0.1 * torch.randn((P,), generator=gen, device="cuda")
        state["x"] = _rows(N, P, pad, TYPES[case["x"]]).copy_(x)
        state["gamma"] = (1.0 + 0.2 * torch.randn((P,), generator=gen, device="cuda")).to(TYPES[case["w"]])
        if op == "layer_norm":
            state["beta"] = (0.1 * torch.randn((P,), generator=gen, device="cuda")).to(TYPES[case["w"]])
            state["type"], state["stats"] = TYPES[case["y"]], case["stats"]
        else:
            # what the forward pass kept, and the gradient that the head sends back
            x = state["x"].double()
            state["mean"] = x.mean(1).float()
            state["rstd"] = (x.var(1, correction=0) + EPS).rsqrt().float()
            state["dy"] = _rows(N, P, pad, TYPES[case["y"]]).copy_(0.05 * torch.randn((N, P), generator=gen, device="cuda"))
        return state
    sizes = _sizes(case)
    total = sum(sizes)
    flat = torch.randn((total,), generator=gen, device="cuda")
    flat *= case["scale"] / math.sqrt(total)
    flat = flat.to(TYPES[case["g"]])
    if case["kind"] == "kernels":
        state["grads"] = [t.clone() for t in flat.split(sizes)]
    else:
        state["grads"] = list(flat.split(sizes))
    if op == "clip_grad_norm":
        # the clipped gradient goes to the optimiser's own buffer, the raw one stays
        state["out"] = torch.empty((total,), dtype=TYPES[case["to"]], device="cuda")
        state["outs"] = list(state["out"].split(sizes))
    return state


def _layer_norm(state):
    x = state["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    y = (d * rstd * state["gamma"].float() + state["beta"].float()).to(state["type"])
    return (y, mean[:, 0], rstd[:, 0]) if state["stats"] else (y, None, None)


def _layer_norm_backward(state):
    dy, mean, rstd = state["dy"].float(), state["mean"][:, None], state["rstd"][:, None]
    xh = (state["x"].float() - mean) * rstd
    u = dy * state["gamma"].float()
    dx = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    w = state["gamma"].dtype
    return dx.to(state["x"].dtype), (dy * xh).sum(0).to(w), dy.sum(0).to(w)


def _grad_norm(grads):
    # many values of one sign: the sums are long
    squares = [g.float().square().sum(dtype=torch.float64) for g in grads]
    return torch.stack(squares).sum().sqrt().float().reshape(1)


def _clip_grad_norm(state):
    norm = _grad_norm(state["grads"])
    c = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    out = torch.cat([(g.float() * c).to(state["out"].dtype) for g in state["grads"]], out=state["out"])
    return norm, out


def run(state):
    op = state["op"]
    if own:
        import paper_2301_08527_b200 as rk
        if op == "layer_norm":
            y, mean, rstd = rk.rocket_layer_norm(state["x"], state["gamma"], state["beta"], EPS, out_dtype=state["type"], want_stats=state["stats"])
            return {"y": y, "mean": mean, "rstd": rstd}
        if op == "layer_norm_backward":
            dx, dgamma, dbeta = rk.rocket_layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["gamma"])
            return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        if op == "grad_norm":
            return {"norm": rk.rocket_grad_norm(state["grads"])}
        norm, _ = rk.rocket_clip_grad_norm(state["grads"], MAX_NORM, out=state["outs"])
        return {"norm": norm, "out": state["out"]}
    if op == "layer_norm":
        y, mean, rstd = _layer_norm(state)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "layer_norm_backward":
        dx, dgamma, dbeta = _layer_norm_backward(state)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "grad_norm":
        return {"norm": _grad_norm(state["grads"])}
    norm, out = _clip_grad_norm(state)
    return {"norm": norm, "out": out}


def work(case):
    """Every input read once and every output written once; a value costs a handful of operations."""
    op = case["op"]
    if op.startswith("layer_norm"):
        N, P = case["N"], case["P"]
        x, y, w = BYTES[case["x"]], BYTES[case["y"]], BYTES[case["w"]]
        if op == "layer_norm":
            return {"bytes": float(N) * P * (x + y) + 2.0 * P * w + (8.0 * N if case["stats"] else 0.0), "flops": 8.0 * N * P}
        return {"bytes": float(N) * P * (2 * x + y) + 8.0 * N + 3.0 * P * w, "flops": 16.0 * N * P}
    total = float(sum(_sizes(case)))
    if op == "grad_norm":
        return {"bytes": total * BYTES[case["g"]] + 4.0, "flops": 2.0 * total}
    return {"bytes": total * (BYTES[case["g"]] + BYTES[case["to"]]) + 4.0, "flops": 3.0 * total}


def exact(case, seed):
    """The same from the definitions, in 64 bits."""
    state = prepare(case, seed)
    op = case["op"]
    f64 = torch.float64
    if op == "layer_norm":
        x = state["x"].to(f64)
        mu = x.sum(dim=-1) / case["P"]
        x.sub_(mu.unsqueeze(-1))
        r = (torch.linalg.vector_norm(x, dim=-1).square() / case["P"] + EPS) ** -0.5
        x.mul_(r.unsqueeze(-1)).mul_(state["gamma"].to(f64)).add_(state["beta"].to(f64))
        return {"y": x, "mean": mu if case["stats"] else None, "rstd": r if case["stats"] else None}
    if op == "layer_norm_backward":
        m, r, g = state["mean"].to(f64), state["rstd"].to(f64), state["gamma"].to(f64)
        xh = torch.addcmul(-(m * r).unsqueeze(-1), state["x"].to(f64), r.unsqueeze(-1))
        dy = state["dy"].to(f64)
        dgamma, dbeta = torch.einsum("np,np->p", dy, xh), torch.einsum("np->p", dy)
        c1, c2 = dy @ g / case["P"], torch.einsum("np,np,p->n", dy, xh, g) / case["P"]
        dx = (dy * g).sub_(c1.unsqueeze(-1)).sub_(xh.mul_(c2.unsqueeze(-1))).mul_(r.unsqueeze(-1))
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    flat = torch.cat([t.reshape(-1) for t in state["grads"]]).to(f64)
    n = torch.linalg.vector_norm(flat)
    if op == "grad_norm":
        return {"norm": n.reshape(1)}
    return {"norm": n.reshape(1), "out": flat * min(1.0, MAX_NORM / (float(n) + 1e-6))}
