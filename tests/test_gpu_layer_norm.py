"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and h half a step of the output's type.  A thread adds at most 32 values in two
chains, 16 more additions join it to its warp, block and cluster: a sum over a row passes fewer than 40 roundings and is off by at
most 40 u of the sum of magnitudes.  Where the rows are not far from zero, their mean (of values of up to |m| + s, with s the
standard deviation) is off by at most 40 u (|m| + s), which is 80 u in units of s while |m| <= s; rows far from zero are taken
relative to their first value.  r is off by 20 u through the variance's 40 u and by 8 u through the roundings of a difference, two
products and the root: 48 u holds both.  A sum over rows may be taken in any order: N u of the sum of magnitudes.
"""
import numpy as np
import pytest

import paper_2301_08527_b200 as rk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


def _torch():
    import torch
    return torch


def _type(name):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _half(dtype):
    torch = _torch()
    return torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def _rows(rng, N, P, dtype, pad, loc=0.0, scale=1.0):
    torch = _torch()
    buf = torch.full((N, P + pad), 7.0, dtype=dtype, device="cuda")
    v = buf[:, :P]
    v.copy_(torch.from_numpy((loc + scale * rng.normal(size=(N, P))).astype(np.float32)))
    return v


def _vec(rng, P, dtype, loc):
    return _torch().from_numpy((loc + 0.5 * rng.normal(size=P)).astype(np.float32)).to(dtype).cuda()


def _d(t):
    return t.double().cpu().numpy()


def _reference(x, g, b, eps):
    m = x.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt(((x - m) ** 2).mean(axis=1, keepdims=True) + eps)
    xh = (x - m) * r
    return xh, xh * g + b, m[:, 0], r[:, 0]


def _check_forward(x, gamma, beta, eps, y, mean, rstd):
    N, P = x.shape
    g = _d(gamma) if gamma is not None else np.ones(P)
    b = _d(beta) if beta is not None else np.zeros(P)
    xh, ref, m, r = _reference(_d(x), g, b, np.float64(np.float32(eps)))
    h, floor = _half(y.dtype)
    own = U * (48 * np.abs(xh * g) + 80 * np.abs(g) + 2 * np.abs(b))
    err = np.abs(_d(y) - ref)
    tol = own * (1 + h) + h * np.abs(ref) + floor
    assert np.all(err <= tol), (float((err / tol).max()), np.unravel_index(np.argmax(err / tol), err.shape))
    if mean is not None:
        # the mean of values that spread by 1 / r about it
        assert np.all(np.abs(_d(mean) - m) <= 2 * U * np.abs(m) + 80 * U / r)
    if rstd is not None:
        assert np.all(np.abs(_d(rstd) - r) <= 48 * U * r)


LENGTHS = [1, 2, 3, 7, 8, 31, 32, 33, 100, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 5000,
           8191, 8192, 8193, 9996, 16384, 16389, 20000, 32768, 32771, 50001, 65536, 65539, 131072, 131075, 300001]


@pytest.mark.parametrize("P", LENGTHS)
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f16", "f32"), ("f16", "f32", "bf16")])
def test_forward_lengths(P, x, y, w):
    rng = np.random.default_rng(P)
    for N, pad in [(1, 0), (3, 5)] + ([(40, 8)] if P < 20000 else []):
        feat, g, b = _rows(rng, N, P, _type(x), pad, 0.7, 1.3), _vec(rng, P, _type(w), 1.0), _vec(rng, P, _type(w), 0.0)
        out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS, out_dtype=_type(y))
        _check_forward(feat, g, b, EPS, out, mean, rstd)


@pytest.mark.parametrize("N,P", [(2, 64), (147, 300), (148, 1024), (149, 1025), (297, 2500), (600, 4096), (1200, 515), (5000, 40), (20011, 9), (70001, 3), (32, 20000),
                                 (200, 20000), (300, 9996), (150, 33000)])
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("f16", "f16", "f16"), ("bf16", "f32", "f32")])
def test_forward_batches(N, P, x, y, w):
    rng = np.random.default_rng(N + P)
    feat, g, b = _rows(rng, N, P, _type(x), 0, -0.3, 2.0), _vec(rng, P, _type(w), 1.0), _vec(rng, P, _type(w), 0.0)
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS, out_dtype=_type(y))
    _check_forward(feat, g, b, EPS, out, mean, rstd)


@pytest.mark.parametrize("P", [5, 300, 2000, 20000, 200003])
@pytest.mark.parametrize("gamma,beta", [(False, False), (True, False), (False, True)])
def test_forward_without_gain_or_bias(P, gamma, beta):
    rng = np.random.default_rng(P)
    feat = _rows(rng, 5, P, _type("f32"), 0)
    g = _vec(rng, P, _type("f16"), 1.0) if gamma else None
    b = _vec(rng, P, _type("bf16"), 0.0) if beta else None
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, want_stats=False)
    assert mean is None and rstd is None
    _check_forward(feat, g, b, EPS, out, None, None)


@pytest.mark.parametrize("P", [40, 1000, 3000, 20000, 70000, 300001])
@pytest.mark.parametrize("loc,scale", [(1000.0, 1e-3), (-3e5, 1.0), (30.0, 1.0), (0.0, 1e-12), (1e-3, 1e-20)])
def test_rows_far_from_zero_and_of_any_scale(P, loc, scale):
    # differences from a value next to the mean are exact where the spread is far below it
    rng = np.random.default_rng(P)
    feat, g, b = _rows(rng, 4, P, _type("f32"), 3, loc, scale), _vec(rng, P, _type("f32"), 1.0), _vec(rng, P, _type("f32"), 0.0)
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS)
    _check_forward(feat, g, b, EPS, out, mean, rstd)


@pytest.mark.parametrize("P", [1, 6, 129, 2000, 20000, 100001])
def test_constant_rows_give_the_bias(P):
    torch = _torch()
    for v in (0.0, 1.0, -3.7, 1e30):
        feat = torch.full((3, P), v, device="cuda")
        rng = np.random.default_rng(P)
        g, b = _vec(rng, P, torch.float32, 1.0), _vec(rng, P, torch.float32, 0.0)
        out, mean, rstd = rk.rocket_layer_norm(feat, g, b, 1e-5)
        assert torch.equal(out, b.expand(3, P)) and torch.equal(mean, feat[:, 0])
        assert np.allclose(_d(rstd), 1e-5 ** -0.5, rtol=8 * U + 1e-7)


@pytest.mark.parametrize("P", [3, 200, 1500, 9996, 20000, 140001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_bad_value_stays_in_its_row(P, bad):
    torch = _torch()
    rng = np.random.default_rng(P)
    feat, g, b = _rows(rng, 9, P, torch.float32, 0), _vec(rng, P, torch.float32, 1.0), _vec(rng, P, torch.float32, 0.0)
    clean = rk.rocket_layer_norm(feat, g, b)
    feat[4, P // 2] = bad
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b)
    rest = [0, 1, 2, 3, 5, 6, 7, 8]
    assert torch.isnan(out[4]).all()
    for got, want in zip((out, mean, rstd), clean):
        assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("P", [1, 7, 64, 257, 1500, 4096, 20000, 70001])
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("f32", "bf16"), ("f16", "f16")])
def test_padding_stays_and_offsets_do_not_matter(P, x, y):
    torch = _torch()
    rng = np.random.default_rng(P)
    N = 6
    g, b = _vec(rng, P + 3, torch.float32, 1.0)[3:], _vec(rng, P + 1, torch.float32, 0.0)[1:]
    feat = _rows(rng, N, P, _type(x), 0)
    want, wm, wr = rk.rocket_layer_norm(feat, g.clone(), b.clone(), out_dtype=_type(y))
    for at, pad in [(1, 0), (3, 1), (8, 8), (0, 13)]:
        buf = torch.full((at + N * (P + pad) + 64,), 5.0, dtype=_type(x), device="cuda")
        fx = buf[at:at + N * (P + pad)].view(N, P + pad)[:, :P]
        fx.copy_(feat)
        obuf = torch.full((at + N * (P + pad) + 64,), 9.0, dtype=_type(y), device="cuda")
        fy = obuf[at:at + N * (P + pad)].view(N, P + pad)[:, :P]
        rk.rocket_layer_norm(fx, g, b, out=fy)
        h, _ = _half(_type(y))
        assert torch.allclose(fy.double(), want.double(), rtol=0, atol=0) or np.all(
            np.abs(_d(fy) - _d(want)) <= 2 * h * np.abs(_d(want)) + 260 * U * (1 + np.abs(_d(g)) * 9))
        rest = obuf.clone()
        rest[at:at + N * (P + pad)].view(N, P + pad)[:, :P] = 9.0
        assert torch.all(rest == 9.0)


def test_interleaved_halves_of_one_buffer_and_a_repeated_row():
    torch = _torch()
    rng = np.random.default_rng(2)
    both = torch.zeros((50, 600), device="cuda")
    both[:, :300] = _rows(rng, 50, 300, torch.float32, 0)
    keep = both[:, :300].clone()
    rk.rocket_layer_norm(both[:, :300], out=both[:, 300:])
    assert torch.equal(both[:, :300], keep)
    _check_forward(keep, None, None, EPS, both[:, 300:], None, None)
    one = _rows(rng, 1, 300, torch.float32, 0)
    out, _, _ = rk.rocket_layer_norm(one.expand(7, 300))
    assert torch.equal(out, rk.rocket_layer_norm(one)[0].expand(7, 300)) or np.allclose(_d(out), _d(rk.rocket_layer_norm(one)[0]), atol=160 * U * 5)
    _check_forward(one.expand(7, 300), None, None, EPS, out, None, None)


def test_other_shapes_and_no_rows():
    torch = _torch()
    rng = np.random.default_rng(3)
    x = _rows(rng, 24, 70, torch.float32, 0)
    want = rk.rocket_layer_norm(x)
    got = rk.rocket_layer_norm(x.view(2, 3, 4, 70))
    assert got[0].shape == (2, 3, 4, 70) and got[1].shape == (2, 3, 4)
    assert torch.equal(got[0].view(24, 70), want[0]) and torch.equal(got[2].view(24), want[2])
    y, m, r = rk.rocket_layer_norm(x[0])
    assert y.shape == (70,) and m.shape == ()
    _check_forward(x[:1], None, None, EPS, y[None], m[None], r[None])
    y, m, r = rk.rocket_layer_norm(torch.empty((0, 5), device="cuda"))
    assert y.shape == (0, 5) and m.shape == (0,)
    w = torch.ones(5, device="cuda")
    dx, dg, db = rk.rocket_layer_norm_backward(y, torch.empty((0, 5), device="cuda"), m, r, w)
    assert dx.shape == (0, 5) and torch.equal(dg, torch.zeros_like(w)) and torch.equal(db, torch.zeros_like(w))


# rows on every alignment (odd lengths and distances), many for each owner, so that stages are used again and again
MANY = [(12000, 515, 0), (9000, 516, 2), (7000, 1001, 0), (3000, 2001, 1), (2600, 4095, 0), (2000, 4097, 3), (1500, 5003, 0), (700, 9996, 6), (700, 10002, 0), (500, 20001, 1),
        (400, 20004, 0), (60000, 100, 1), (50000, 257, 0), (30000, 300, 5), (20000, 511, 0)]


@pytest.mark.parametrize("N,P,pad", MANY)
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("f32", "f16", "f16")])
def test_forward_many_rows_of_any_alignment(N, P, pad, x, y, w):
    rng = np.random.default_rng(N + P)
    feat, g, b = _rows(rng, N, P, _type(x), pad, 0.4, 1.5), _vec(rng, P, _type(w), 1.0), _vec(rng, P, _type(w), 0.0)
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS, out_dtype=_type(y))
    _check_forward(feat, g, b, EPS, out, mean, rstd)


@pytest.mark.parametrize("N,P,pad", MANY)
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("f32", "f16", "f16")])
def test_backward_many_rows_of_any_alignment(N, P, pad, x, y, w):
    rng = np.random.default_rng(N + P + 1)
    feat, dy = _rows(rng, N, P, _type(x), pad, 0.4, 1.5), _rows(rng, N, P, _type(y), pad + 3, 0.1, 1.0)
    g, (m, r) = _vec(rng, P, _type(w), 1.0), _stats(feat)
    _check_backward(dy, feat, m, r, g, *rk.rocket_layer_norm_backward(dy, feat, m, r, g))


# ---- backward ------------------------------------------------------------------------------------------------------------

def _check_backward(dy, x, mean, rstd, gamma, dx, dg, db):
    N, P = x.shape
    m, r = _d(mean)[:, None], _d(rstd)[:, None]
    g = _d(gamma) if gamma is not None else np.ones(P)
    d = _d(dy)
    xh = (_d(x) - m) * r
    u = d * g
    c1, c2 = u.mean(axis=1, keepdims=True), (u * xh).mean(axis=1, keepdims=True)
    a1, a2 = np.abs(u).mean(axis=1, keepdims=True), np.abs(u * xh).mean(axis=1, keepdims=True)
    if dx is not None:
        ref = r * (u - c1 - xh * c2)
        h, floor = _half(dx.dtype)
        own = U * r * (6 * np.abs(u) + 4 * np.abs(c1) + 84 * a1 + np.abs(xh) * (8 * np.abs(c2) + 88 * a2))
        err, tol = np.abs(_d(dx) - ref), own * (1 + h) + h * np.abs(ref) + floor
        assert np.all(err <= tol), (float((err / tol).max()), np.unravel_index(np.argmax(err / tol), err.shape))
    for got, terms, k in ((dg, d * xh, 4), (db, d, 1)):
        if got is not None:
            ref = terms.sum(axis=0)
            h, floor = _half(got.dtype)
            err, tol = np.abs(_d(got) - ref), (N + k) * U * np.abs(terms).sum(axis=0) * (1 + h) + h * np.abs(ref) + floor
            assert np.all(err <= tol), (float((err / tol).max()), int(np.argmax(err / tol)))


def _stats(x):
    v = x.double()
    return v.mean(1).float(), (v.var(1, correction=0) + EPS).rsqrt().float()


@pytest.mark.parametrize("P", LENGTHS)
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f16", "f32"), ("f16", "f32", "bf16")])
def test_backward_lengths(P, x, y, w):
    rng = np.random.default_rng(P + 1)
    for N, pad in [(1, 0), (3, 5)] + ([(40, 8)] if P < 20000 else []):
        feat, dy = _rows(rng, N, P, _type(x), pad, 0.7, 1.3), _rows(rng, N, P, _type(y), pad, 0.1, 1.0)
        g, (m, r) = _vec(rng, P, _type(w), 1.0), _stats(feat)
        _check_backward(dy, feat, m, r, g, *rk.rocket_layer_norm_backward(dy, feat, m, r, g))


@pytest.mark.parametrize("N,P", [(2, 64), (147, 300), (148, 1024), (149, 1025), (297, 2500), (600, 4096), (1200, 515), (3000, 40), (3900, 9), (3800, 1), (32, 20000),
                                 (200, 20000), (300, 9996), (150, 33000), (64, 66000), (1500, 2048), (1000, 8192)])
@pytest.mark.parametrize("x,y,w", [("f32", "f32", "f32"), ("f16", "f16", "f16"), ("bf16", "f32", "f32")])
def test_backward_batches(N, P, x, y, w):
    rng = np.random.default_rng(N + P)
    feat, dy = _rows(rng, N, P, _type(x), 0, -0.3, 2.0), _rows(rng, N, P, _type(y), 0, 0.0, 1.0)
    g, (m, r) = _vec(rng, P, _type(w), 1.0), _stats(feat)
    _check_backward(dy, feat, m, r, g, *rk.rocket_layer_norm_backward(dy, feat, m, r, g))


@pytest.mark.parametrize("N,P", [(5, 33), (200, 1000), (7, 20000), (300, 4096), (40, 70001)])
def test_backward_parts_on_their_own(N, P):
    torch = _torch()
    rng = np.random.default_rng(N)
    feat, dy = _rows(rng, N, P, torch.float32, 0), _rows(rng, N, P, torch.float32, 0)
    m, r = _stats(feat)
    g = _vec(rng, P, torch.float32, 1.0)
    for gamma in (g, None):
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, m, r, gamma, want_weights=False)
        assert dg is None and db is None
        _check_backward(dy, feat, m, r, gamma, dx, None, None)
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, m, r, gamma, want_dx=False)
        assert dx is None
        _check_backward(dy, feat, m, r, gamma, None, dg, db)
        out = torch.empty(P, dtype=torch.bfloat16, device="cuda")
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, m, r, None, want_dx=False, want_weights=False, dbeta_out=out)
        assert dx is None and dg is None and db is out
        _check_backward(dy, feat, m, r, None, None, None, db)
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, m, r, gamma, want_weights=False, dgamma_out=torch.empty(P, device="cuda"))
        assert db is None
        _check_backward(dy, feat, m, r, gamma, dx, dg, None)


@pytest.mark.parametrize("P", [2, 65, 300, 2048, 9996, 20000, 70001])
@pytest.mark.parametrize("N", [3, 50, 400])
def test_backward_is_the_same_bits_again_and_leaves_padding(N, P):
    torch = _torch()
    rng = np.random.default_rng(P)
    feat, dy = _rows(rng, N, P, torch.float32, 3), _rows(rng, N, P, torch.bfloat16, 1)
    m, r = _stats(feat)
    g = _vec(rng, P, torch.float32, 1.0)
    buf = torch.full((N, P + 2), 9.0, device="cuda")
    first = None
    for _ in range(3):
        dx, dg, db = rk.rocket_layer_norm_backward(dy, feat, m, r, g, dx_out=buf[:, :P])
        assert torch.all(buf[:, P:] == 9.0)
        got = [dx.clone(), dg, db]
        if first is not None:
            assert all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


def test_backward_of_rows_that_one_row_stands_for():
    # a broadcast input: the gradient of the one row is the sum over its copies, which the caller takes
    torch = _torch()
    rng = np.random.default_rng(8)
    one = _rows(rng, 1, 500, torch.float32, 0)
    feat, dy = one.expand(60, 500), _rows(rng, 1, 500, torch.float32, 0).expand(60, 500)
    m, r = _stats(feat.contiguous())
    _check_backward(dy, feat, m, r, None, *rk.rocket_layer_norm_backward(dy, feat, m, r))


def test_gradients_against_differences():
    # central differences of f = sum(dy * y) in the kernel's own forward, step 2^-6: the truncation is of the order of the
    # third derivative times 2^-12 / 6, fp32 rounding of the terms' sum below 1e-4 of the step
    torch = _torch()
    rng = np.random.default_rng(9)
    N, P, step = 3, 12, 2.0 ** -6
    x, g, b = rng.normal(size=(N, P)), 1 + 0.3 * rng.normal(size=P), rng.normal(size=P)
    dy = rng.normal(size=(N, P))
    dev = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731

    def f(x, g, b):
        return float((dev(dy).double() * rk.rocket_layer_norm(dev(x), dev(g), dev(b))[0].double()).sum())

    _, m, r = rk.rocket_layer_norm(dev(x), dev(g), dev(b))
    got = rk.rocket_layer_norm_backward(dev(dy), dev(x), m, r, dev(g))
    for i, (a, grad) in enumerate(zip((x, g, b), got)):
        grad = _d(grad)
        for at in np.ndindex(a.shape):
            args = []
            for s in (1, -1):
                v = [x.copy(), g.copy(), b.copy()]
                v[i][at] += s * step
                args.append(f(*v))
            assert abs((args[0] - args[1]) / (2 * step) - grad[at]) <= 2e-3, (i, at)


def test_offsets_beyond_32_bits():
    torch = _torch()
    N, P = 70000, 33001                          # 2.3e9 values, rows on every alignment
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn((N, P), generator=gen, device="cuda", dtype=torch.bfloat16)
    g = torch.rand(P, generator=gen, device="cuda") + 0.5
    y, m, r = rk.rocket_layer_norm(x, g)
    some = [0, 1, 32767, 65075, 65076, N - 2, N - 1]
    for n in some:
        _check_forward(x[n:n + 1], g, None, EPS, y[n:n + 1], m[n:n + 1], r[n:n + 1])
    dx, dg, db = rk.rocket_layer_norm_backward(y, x, m, r, g)
    for n in some:
        _check_backward(y[n:n + 1], x[n:n + 1], m[n:n + 1], r[n:n + 1], g, dx[n:n + 1], None, None)
    # the sums over all rows of the columns at both ends, any order: N u of the magnitudes
    for c in (0, P - 1):
        d, xh = _d(y[:, c]), (_d(x[:, c]) - _d(m)) * _d(r)
        assert abs(float(dg[c]) - (d * xh).sum()) <= (N + 4) * U * np.abs(d * xh).sum()
        assert abs(float(db[c]) - d.sum()) <= (N + 1) * U * np.abs(d).sum()


# ---- how a program calls them --------------------------------------------------------------------------------------------

SIZES = [(1, 20000), (32, 20000), (700, 1000), (100, 1000), (5000, 64), (500, 65), (40, 70001)]


@pytest.mark.parametrize("N,P", SIZES)
def test_captured_calls_give_the_bits_of_plain_calls(N, P):
    torch = _torch()
    rng = np.random.default_rng(N)
    feat, dy = _rows(rng, N, P, torch.float32, 0), _rows(rng, N, P, torch.float32, 0)
    g, b = _vec(rng, P, torch.float32, 1.0), _vec(rng, P, torch.float32, 0.0)

    def calls():
        y, m, r = rk.rocket_layer_norm(feat, g, b)
        return (y, m, r) + rk.rocket_layer_norm_backward(dy, feat, m, r, g)

    calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):                      # two graphs that run at the same time share no scratch memory
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = calls()
            graphs.append((graph, out))
    torch.cuda.synchronize()
    for shift in (0.0, 0.5):
        feat += shift * torch.arange(P, device="cuda") / P
        want = calls()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for _ in range(5):
            for (graph, _), s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, c) for a, c in zip(out, want))


@pytest.mark.parametrize("N,P", SIZES)
def test_calls_on_two_streams_at_once(N, P):
    torch = _torch()
    rng = np.random.default_rng(N)
    feat, dy = _rows(rng, N, P, torch.float32, 0), _rows(rng, N, P, torch.float32, 0)
    g = _vec(rng, P, torch.float32, 1.0)
    y, m, r = rk.rocket_layer_norm(feat, g)
    want = (y,) + rk.rocket_layer_norm_backward(dy, feat, m, r, g)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(4)]:
        with torch.cuda.stream(s):
            for _ in range(4):
                got.append((rk.rocket_layer_norm(feat, g)[0],) + rk.rocket_layer_norm_backward(dy, feat, m, r, g))
    torch.cuda.synchronize()
    for one in got:
        assert all(torch.equal(a, b) for a, b in zip(one, want))


def test_nothing_is_allocated_by_the_library_and_kernels_are_counted():
    torch = _torch()
    feat = torch.randn((100, 3000), device="cuda")
    allocs, launches = rk.device_alloc_count(), rk.kernel_launch_count()
    y, m, r = rk.rocket_layer_norm(feat)
    rk.rocket_layer_norm_backward(y, feat, m, r)
    assert rk.device_alloc_count() == allocs and rk.kernel_launch_count() >= launches + 2


def test_refusals_of_the_binding():
    torch = _torch()
    x = torch.randn((6, 8), device="cuda")
    y, m, r = rk.rocket_layer_norm(x)
    w = torch.ones(8, device="cuda")
    for bad in (x.double(), x.int(), x.t(), x[:, ::2], torch.randn((3, 4, 8), device="cuda")[:, :2], torch.tensor(1.0, device="cuda")):
        with pytest.raises(TypeError):
            rk.rocket_layer_norm(bad)
    for kw in (dict(gamma=w[:7]), dict(beta=torch.ones(9, device="cuda")), dict(out=torch.empty((6, 9), device="cuda")), dict(mean_out=torch.empty(5, device="cuda"))):
        with pytest.raises(ValueError):
            rk.rocket_layer_norm(x, **kw)
    for kw in (dict(gamma=w, beta=w.half()), dict(gamma=w.cpu()), dict(out=y.half(), out_dtype=torch.float32), dict(gamma=torch.ones(16, device="cuda")[::2]),
               dict(rstd_out=torch.empty(6, dtype=torch.float16, device="cuda")), dict(out=torch.empty((8, 6), device="cuda").t())):
        with pytest.raises(TypeError):
            rk.rocket_layer_norm(x, **kw)
    with pytest.raises(ValueError):
        rk.rocket_layer_norm(torch.empty((3, 0), device="cuda"))
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(out=x)):
        with pytest.raises(rk.RocketError):
            rk.rocket_layer_norm(x, **kw)
    with pytest.raises(rk.RocketError):
        rk.rocket_layer_norm_backward(y, x, m, r, want_dx=False, want_weights=False)
    with pytest.raises(rk.RocketError):
        rk.rocket_layer_norm_backward(y, x, m, r, dx_out=x)
    with pytest.raises(TypeError):
        rk.rocket_layer_norm_backward(y, x, None, r)
    with pytest.raises(TypeError):
        rk.rocket_layer_norm_backward(y, x, m, r, w, weight_dtype=torch.float16)
    with pytest.raises(ValueError):
        rk.rocket_layer_norm_backward(y[:5], x, m, r)
    with pytest.raises(TypeError):
        rk.rocket_layer_norm_backward(y, x, m, r, w, dgamma_out=w.half())
