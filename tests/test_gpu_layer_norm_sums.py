"""Layer norm backward with inputs of small whole numbers, mean 0 and rstd 1: then dgamma = sum dy x and dbeta = sum dy are whole numbers
below 2^24, which fp32 holds in whatever order they are added, and one lost, doubled or stale row shows in every column."""
import numpy as np
import pytest

import paper_2301_08527_b200 as rk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    return torch


def _type(name):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _whole(gen, N, P, dtype, at, pad, most):
    """[N, P] of -most .. most, the first row `at` values behind a 16-byte border, rows `pad` values apart."""
    torch = _torch()
    buf = torch.empty(at + N * (P + pad), dtype=dtype, device="cuda")
    v = buf[at:].view(N, P + pad)[:, :P]
    v.copy_(torch.randint(-most, most + 1, (N, P), generator=gen, device="cuda"))
    return v


def _unit(N):
    torch = _torch()
    return torch.zeros(N, device="cuda"), torch.ones(N, device="cuda")


def _check_dx(dx, dy, x):
    # as rounded: u = dy, xh = x and the sums over a row are whole and exact; 1/P, two products and two sums of fp32 follow (8 u holds them)
    d, v = dy.double(), x.double()
    c1, c2 = d.mean(1, keepdim=True), (d * v).mean(1, keepdim=True)
    ref = d - c1 - v * c2
    h = _torch().finfo(dx.dtype).eps / 2
    tol = 8 * U * (d.abs() + c1.abs() + (v * c2).abs()) * (1 + h) + h * ref.abs() + 2.0 ** -25
    assert bool(((dx.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("N", [1, 2, 3, 40])
@pytest.mark.parametrize("P", [4097, 5003, 9997, 20003, 33001, 65535])
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "f16"), ("f32", "bf16")])
def test_first_rows_of_every_owner_at_any_alignment(N, P, x, y):
    gen = _torch().Generator(device="cuda")
    gen.manual_seed(P + N)
    for k in range(6):                          # other values each time: what a block's shared memory held before shows
        feat, dy = _whole(gen, N, P, _type(x), k % 4, k, 3), _whole(gen, N, P, _type(y), (k + 1) % 8, 1, 3)
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N))
        assert np.array_equal(dg.double().cpu().numpy(), (dy.double() * feat.double()).sum(0).cpu().numpy())
        assert np.array_equal(db.double().cpu().numpy(), dy.double().sum(0).cpu().numpy())
        _check_dx(dx, dy, feat)


@pytest.mark.parametrize("N,P", [(1, 7), (2, 4096), (5, 600), (16, 1001), (40, 513), (300, 40), (500, 257)])
def test_one_of_the_sums_of_few_rows(N, P):
    torch = _torch()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    for _ in range(20):
        feat, dy = _whole(gen, N, P, torch.float32, 0, 0, 3), _whole(gen, N, P, torch.float32, 0, 0, 3)
        wg, wb = (dy.double() * feat.double()).sum(0).float(), dy.double().sum(0).float()
        _, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N), want_dx=False, want_weights=False, dgamma_out=torch.empty(P, device="cuda"))
        assert db is None and torch.equal(dg, wg)
        _, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N), want_dx=False, want_weights=False, dbeta_out=torch.empty(P, device="cuda"))
        assert dg is None and torch.equal(db, wb)
        _, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N))
        assert torch.equal(dg, wg) and torch.equal(db, wb)


@pytest.mark.parametrize("N,P", [(1, 5), (4, 1000), (20, 1000), (128, 1001), (128, 4096), (64, 4095), (4096, 128), (4097, 128), (2048, 256), (1024, 512), (1, 20000), (3, 20000)])
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16")])
def test_dx_alone_has_the_bits_of_dx_with_the_sums(N, P, x, y):
    torch = _torch()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    feat, dy = _whole(gen, N, P, _type(x), 0, 0, 3), _whole(gen, N, P, _type(y), 0, 0, 3)
    dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N), want_weights=False)
    assert dg is None and db is None
    _check_dx(dx, dy, feat)
    assert torch.equal(dx, rk.rocket_layer_norm_backward(dy, feat, *_unit(N))[0])


def _check_whole_sums(N, P, x, y, at, pad, low, most):
    """dgamma and dbeta to the bit: sums over up to an eighth of the rows stay below 2^24 and are exact in fp32, the whole's are rounded to fp32 once."""
    torch = _torch()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + P)
    feat, dy = _whole(gen, N, P, _type(x), at, pad, 2), _whole(gen, N, P, _type(y), at, pad, most)
    if low is not None:                         # of one sign
        feat.copy_(feat.abs() + 1)
        dy.copy_(dy.abs().clamp(min=low))
    dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, *_unit(N))
    # whole sums of up to 2^53: exact in double, by columns to spare memory
    for lo in range(0, P, 256):
        d, v = dy[:, lo:lo + 256].double(), feat[:, lo:lo + 256].double()
        assert torch.equal(dg[lo:lo + 256], (d * v).sum(0).float()) and torch.equal(db[lo:lo + 256], d.sum(0).float())
    return dx, dy, feat


# one row and more above what 16 blocks join, for 8, 16 and 32 lanes and for blocks and clusters; on and off 16-byte borders: words of 8, 4 and 1
ABOVE = [(4097, 64), (4111, 128), (5000, 100), (4999, 97), (2049, 136), (2500, 200), (2499, 256), (2100, 251), (1025, 264), (1500, 320), (1499, 512), (1100, 505), (129, 520),
         (300, 1000), (299, 1001), (150, 4096), (20, 4104), (400, 9996), (77, 20000), (40, 33001)]


@pytest.mark.parametrize("N,P", ABOVE + [(4096, 128), (2048, 256), (1024, 512), (128, 4096), (3000, 96), (500, 300), (100, 1003)])
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("at,pad", [(0, 0), (1, 0), (0, 8)])
def test_every_row_counts_once(N, P, x, y, at, pad):
    dx, dy, feat = _check_whole_sums(N, P, x, y, at, pad, None, 3)
    _check_dx(dx, dy, feat)


@pytest.mark.parametrize("N,P", [(70001, 64), (50000, 200), (40001, 257), (30000, 512), (20000, 1000), (12000, 4096), (12001, 4099), (8000, 9996), (4096, 128), (2000, 256), (128, 4096)])
def test_long_sums_of_one_sign_are_rounded_once(N, P):
    # dy of about 3/4 of most and x of 2.2 in the mean: sums of about 2^26, 1.65 most N, of which an eighth is below 2^24
    most = int(2 ** 26 / (1.65 * N))
    _check_whole_sums(N, P, "f32", "f32", 0, 0, most // 2, most)
