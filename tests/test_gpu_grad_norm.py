"""Gradient norm and clipping against their definition in 64 bits.

Squares and sums are double: the norm is off by the rounding to fp32, u = 2^-24, and by less than 2^-40.  The factor c adds
the roundings of norm + 1e-6, of the quotient and of the product (3 u), the output half a step of its type.
"""
import math

import numpy as np
import pytest

import paper_2301_08527_b200 as rk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    return torch


def _grads(sizes, types, seed=0, scale=1.0):
    torch = _torch()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kinds = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
    return [(scale * torch.randn((n,), generator=gen, device="cuda")).to(kinds[types[i % len(types)]]) for i, n in enumerate(sizes)]


def _norm(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def _check(before, norm, max_norm, after):
    torch = _torch()
    ref = _norm(before)
    assert abs(float(norm) - ref) <= (U + 2 ** -40) * ref
    c = min(1.0, max_norm / (ref + 1e-6))
    for g, o in zip(before, after):
        if not g.numel():
            continue
        h, floor = torch.finfo(o.dtype).eps / 2, torch.finfo(o.dtype).smallest_normal * torch.finfo(o.dtype).eps / 2
        want = g.double() * c
        assert bool(((o.double() - want).abs() <= (5 * U + h) * want.abs() * (1 + 5 * U) + floor).all())


MIXES = [[1], [3], [1000], [1023, 1024, 1025], [16384], [16385], [16383, 1, 16384, 7, 40000], [100000], [0, 5, 0], [1 << 20, 3, 77], [5000000, 12345],
         list(range(0, 130)), [17] * 500, [300000 + i for i in range(20)], [2000003, 1, 1999999]]


@pytest.mark.parametrize("sizes", MIXES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("types", [("f32",), ("f16",), ("bf16",), ("f32", "bf16", "f16")], ids="_".join)
def test_norm_and_clipping(sizes, types):
    torch = _torch()
    grads = _grads(sizes, types, len(sizes))
    ref = _norm(grads)
    assert abs(float(rk.rocket_grad_norm(grads)) - ref) <= (U + 2 ** -40) * ref
    for max_norm in (0.3 * ref, 10.0 * ref + 1.0):
        keep = [g.clone() for g in grads]
        # into other tensors, of the same type and of fp32
        for wide in (False, True):
            out = [torch.full_like(g, 9.0, dtype=torch.float32 if wide else g.dtype) for g in grads]
            norm, got = rk.rocket_clip_grad_norm(grads, max_norm, out=out)
            assert got is out and all(torch.equal(a, b) for a, b in zip(keep, grads))
            _check(keep, norm, max_norm, out)
        # in place
        mine = [g.clone() for g in grads]
        norm, got = rk.rocket_clip_grad_norm(mine, max_norm)
        assert got is mine
        _check(keep, norm, max_norm, mine)
        if max_norm > ref:
            assert all(torch.equal(a, b) for a, b in zip(keep, mine))


@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("g,o", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")])
def test_any_alignment_and_the_neighbours_stay(offset, g, o):
    torch = _torch()
    kinds = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
    sizes = [1, 2, 5, 9, 100, 16384, 16391, 33000, 70001]
    total = sum(sizes) + offset * (len(sizes) + 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(offset)
    src = torch.randn((total,), generator=gen, device="cuda").to(kinds[g])
    for shift in (0, 1, 4):                     # the output's alignment against the gradient's
        dst = torch.full((total + shift,), 9.0, dtype=kinds[o], device="cuda")
        at, grads, outs = offset, [], []
        mask = torch.ones(total + shift, dtype=torch.bool, device="cuda")
        for n in sizes:
            grads.append(src[at:at + n])
            outs.append(dst[at + shift:at + shift + n])
            mask[at + shift:at + shift + n] = False
            at += n + offset
        norm, _ = rk.rocket_clip_grad_norm(grads, 1.0, out=outs)
        _check(grads, norm, 1.0, outs)
        assert bool((dst[mask] == 9.0).all())
    keep, mine = src.clone(), src.clone()
    at, grads, mask = offset, [], torch.ones(total, dtype=torch.bool, device="cuda")
    for n in sizes:
        grads.append(mine[at:at + n])
        mask[at:at + n] = False
        at += n + offset
    before = [t.clone() for t in grads]
    norm, _ = rk.rocket_clip_grad_norm(grads, 1.0)
    _check(before, norm, 1.0, grads)
    assert torch.equal(mine[mask], keep[mask])


@pytest.mark.parametrize("value", [1e-30, 1e-22, 3e-39, 1e-45, 1e19, 1e30, 3e38])
@pytest.mark.parametrize("n", [1, 7, 1000, 300001])
def test_values_whose_squares_leave_single_precision(value, n):
    torch = _torch()
    v = np.float32(value)
    g = torch.full((n,), float(v), device="cuda")
    ref = float(v) * math.sqrt(n)
    norm = float(rk.rocket_grad_norm([g]))
    if ref > 3.4028235677973366e38:
        assert math.isinf(norm)
    else:
        assert abs(norm - ref) <= 2 * U * ref + 2.0 ** -150


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 50000])
def test_zeros_infinities_and_nan(t, n):
    torch = _torch()
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[t]
    zero = torch.zeros(n, dtype=kind, device="cuda")
    norm, _ = rk.rocket_clip_grad_norm([zero], 1.0)
    assert float(norm) == 0.0 and bool((zero == 0).all())
    for bad in (float("inf"), float("-inf"), float("nan")):
        g = torch.ones(n, dtype=kind, device="cuda")
        h = torch.ones(33, dtype=kind, device="cuda")
        g[n // 2] = bad
        assert math.isnan(float(rk.rocket_grad_norm([g]))) if math.isnan(bad) else math.isinf(float(rk.rocket_grad_norm([g])))
        norm, _ = rk.rocket_clip_grad_norm([g, h], 1.0)
        if math.isnan(bad):
            assert math.isnan(float(norm)) and bool(torch.isnan(h).all()) and bool(torch.isnan(g).all())
        else:                                   # 1 / inf = 0, and 0 times an infinity is NaN
            rest = torch.ones(n, dtype=torch.bool, device="cuda")
            rest[n // 2] = False
            assert math.isinf(float(norm)) and bool((h == 0).all()) and bool((g[rest] == 0).all()) and bool(torch.isnan(g[n // 2]))
    g = torch.ones(n, dtype=kind, device="cuda")
    rk.rocket_clip_grad_norm([g], 0.0)
    assert bool((g == 0).all())
    g = torch.ones(n, dtype=kind, device="cuda")
    rk.rocket_clip_grad_norm([g], float("inf"))
    assert bool((g == 1).all())


def test_lists_other_shapes_and_repeats():
    torch = _torch()
    assert float(rk.rocket_grad_norm([])) == 0.0
    norm, got = rk.rocket_clip_grad_norm([], 1.0)
    assert float(norm) == 0.0 and got == []
    a = torch.randn((30, 40), device="cuda")
    keep = a.clone()
    t = torch.randn((5, 6, 7, 8), device="cuda").to(memory_format=torch.channels_last)
    ref = _norm([a, t])
    grads = (a.t(), t)                          # dense in another order
    norm, _ = rk.rocket_clip_grad_norm(grads, 0.5)
    assert abs(float(norm) - ref) <= 2 * U * ref
    assert torch.allclose(a, keep * (0.5 / (ref + 1e-6)), rtol=8 * U)
    twice = _norm([keep, keep])
    assert abs(float(rk.rocket_grad_norm([keep, keep])) - twice) <= 2 * U * twice
    with pytest.raises(rk.RocketError):
        rk.rocket_clip_grad_norm([keep, keep], 1.0)
    out = torch.full((1,), 5.0, device="cuda")
    assert rk.rocket_grad_norm([keep], norm_out=out) is out


@pytest.mark.parametrize("count,size", [(3, 100), (40, 70000), (700, 300), (4, 3000000)])
def test_captured_concurrent_and_the_same_bits_again(count, size):
    torch = _torch()
    grads = _grads([size + i for i in range(count)], ("f32", "bf16"), count)
    outs = [[torch.empty_like(g) for g in grads] for _ in range(2)]
    want, _ = rk.rocket_clip_grad_norm(grads, 1.0, out=outs[0])
    want_out = [o.clone() for o in outs[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for k in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                norm, _ = rk.rocket_clip_grad_norm(grads, 1.0, out=outs[k])
                alone = rk.rocket_grad_norm(grads)
            graphs.append((graph, norm, alone))
    torch.cuda.synchronize()
    for o in outs[0] + outs[1]:
        o.fill_(7.0)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for (graph, _, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for (_, norm, alone), out in zip(graphs, outs):
        assert torch.equal(norm, want) and torch.equal(alone, want)
        assert all(torch.equal(a, b) for a, b in zip(out, want_out))


def test_a_tensor_of_more_values_than_32_bits_count():
    torch = _torch()
    n = (1 << 32) + 12345
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    ref = 0.5 * math.sqrt(n)
    norm, _ = rk.rocket_clip_grad_norm([g, torch.zeros(7, device="cuda")], ref / 2)
    assert abs(float(norm) - ref) <= 2 * U * ref
    # 0.25 up to the 1e-6 beside the norm and fp32's roundings: the nearest bfloat16 value
    assert float(g.min()) == 0.25 and float(g.max()) == 0.25


def test_refusals_of_the_binding():
    torch = _torch()
    g = torch.randn((6, 8), device="cuda")
    for bad in ([g.double()], [g.cpu()], [g[:, :4]], [None], [g.expand(2, 6, 8)]):
        with pytest.raises(TypeError):
            rk.rocket_grad_norm(bad)
        with pytest.raises(TypeError):
            rk.rocket_clip_grad_norm(bad, 1.0)
    for out in ([g.clone(), g.clone()], [g.t().clone()], [torch.empty((8, 6), device="cuda").t()], []):
        with pytest.raises(ValueError):
            rk.rocket_clip_grad_norm([g], 1.0, out=out)
    for kw in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=1.0, out=[g.half()])):
        with pytest.raises(rk.RocketError):
            rk.rocket_clip_grad_norm([g], **kw)
    with pytest.raises(TypeError):
        rk.rocket_grad_norm([g], norm_out=torch.zeros(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        rk.rocket_grad_norm([g], norm_out=torch.zeros(2, device="cuda"))
