"""Clipping into lists whose tensors are dense in various orders."""
import math

import pytest

import paper_2301_08527_b200 as rk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_each_pair_of_tensors_has_its_own_order():
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = [torch.randn((30, 40), generator=gen, device="cuda").t(), torch.randn((6, 8), generator=gen, device="cuda"),
             torch.empty_strided((5, 1, 6), (1, 777, 5), device="cuda").normal_(generator=gen)]
    out = [torch.empty((30, 40), device="cuda").t(), torch.empty(48, device="cuda"), torch.empty_strided((5, 1, 6), (1, 5, 5), device="cuda")]
    ref = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    norm, got = rk.rocket_clip_grad_norm(grads, 0.5, out=out)
    assert got is out and abs(float(norm) - ref) <= 2 * U * ref
    for g, o in zip(grads, out):
        want = g.double() * (0.5 / (ref + 1e-6))
        assert bool(((o.double().reshape(want.shape) - want).abs() <= 8 * U * want.abs()).all())
    for bad in ([out[0].contiguous(), out[1], out[2]], [out[0], torch.empty((8, 6), device="cuda").t(), out[2]]):
        with pytest.raises(ValueError):
            rk.rocket_clip_grad_norm(grads, 0.5, out=bad)
