"""Layer norm of rows some of whose values are unlike the others, wherever these lie.

Tolerances are those of test_gpu_layer_norm.py, which hold for these rows too (u = 2^-24, s the row's standard deviation, P >= 20,000 the
hardest): a thread adds up to 32 differences to its first value and is off by 21 u of their mean size; that is 1.2 s for ordinary values, and
where the first value is one of up to three that lie D away, the thread's mean counts 32 / P: 21 u D 32 / P <= 5 u s, as s >= D / sqrt(P).
Joining adds three levels of 8 roundings of the sets' distances from one another, about s each.  A value's distance from its thread's mean is
rounded once: u (|x - m| + 3 D / 32), and D / s <= sqrt(P) keeps the second part below 15 u s up to 320,000 values.  Together less than 80 u s
besides what is proportional to |x - m|.
"""
import numpy as np
import pytest

import paper_2301_08527_b200 as rk
from test_gpu_layer_norm import EPS, _check_forward, _torch, _type, _vec

pytestmark = pytest.mark.gpu

U = 2.0 ** -24

# what is put where, on rows N(loc, 1)
ROWS = {
    "first three large": (0.0, lambda x: x.__setitem__((slice(None), slice(0, 3)), 100.0 + x[:, :3])),
    "first unlike a row far from zero": (1000.0, lambda x: x.__setitem__((slice(None), 0), 0.0)),
    "first and last zero": (1000.0, lambda x: x.__setitem__((slice(None), [0, -1]), 0.0)),
    "first, middle and last large": (0.0, lambda x: x.__setitem__((slice(None), [0, x.shape[1] // 2, -1]), 100.0)),
    "first negative and large": (0.0, lambda x: x.__setitem__((slice(None), 0), -100.0)),
}


@pytest.mark.parametrize("P", [3, 40, 257, 1500, 2049, 4096, 20000, 20003, 81000, 131072, 320000])
@pytest.mark.parametrize("kind", ROWS)
@pytest.mark.parametrize("N,x", [(3, "f32"), (40, "f32"), (3, "f16")])
def test_values_unlike_the_rest(N, x, kind, P):
    torch = _torch()
    rng = np.random.default_rng(P)
    loc, put = ROWS[kind]
    v = loc + rng.normal(size=(N, P))
    put(v)
    feat = torch.from_numpy(v.astype(np.float32)).to(_type(x)).cuda()
    g, b = _vec(rng, P, torch.float32, 1.0), _vec(rng, P, torch.float32, 0.0)
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS, out_dtype=torch.float32)
    _check_forward(feat, g, b, EPS, out, mean, rstd)


@pytest.mark.parametrize("N,P", [(1300, 4096), (2500, 2001), (700, 20000), (300, 50001), (40000, 100)])
@pytest.mark.parametrize("kind", ROWS)
def test_values_unlike_the_rest_in_many_rows(N, P, kind):
    torch = _torch()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(P)
    loc, put = ROWS[kind]
    feat = loc + torch.randn((N, P), generator=gen, device="cuda")
    put(feat)
    out, mean, rstd = rk.rocket_layer_norm(feat)
    _check_forward(feat, None, None, EPS, out, mean, rstd)


@pytest.mark.parametrize("P", [2, 40, 257, 1500, 2049, 4096, 20000, 20003, 81000, 131072, 320000, 400001])
@pytest.mark.parametrize("low,high", [(1e35, 3e35), (1e37, 3e37), (-1e38, 2e38), (2e38, 3.4e38), (-3.4e38, -3.3e38)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_finite_rows_at_the_ends_of_the_range(x, low, high, P):
    torch = _torch()
    rng = np.random.default_rng(P)
    feat = torch.from_numpy(rng.uniform(low, high, size=(3, P))).to(_type(x)).cuda()
    if x == "bf16":
        feat = feat.clamp(-3.38e38, 3.38e38)
    assert bool(torch.isfinite(feat).all())
    g, b = _vec(rng, P, torch.float32, 1.0), _vec(rng, P, torch.float32, 0.0)
    out, mean, rstd = rk.rocket_layer_norm(feat, g, b, EPS, out_dtype=torch.float32)
    v = feat.double()
    m, s = v.mean(1), v.std(1, correction=0)
    assert bool(((mean.double() - m).abs() <= 2 * U * m.abs() + 80 * U * s).all())
    zero = rstd == 0
    # 1 / s where doubles sum up the squares (and fp32 still holds it to half a step, 2^-150 where it is subnormal)
    assert bool((zero | ((rstd.double() - 1 / s).abs() <= 48 * U / s + 2.0 ** -149)).all())
    assert torch.equal(out[zero], b.expand(3, P)[zero])
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("P", [40, 1500, 4096, 20000, 20003, 131072, 320000, 400001])
def test_variances_whose_sums_leave_single_precision(P):
    # values within 1e18 of the mean: squares up to 1e36, sums of them up to 3e40
    torch = _torch()
    rng = np.random.default_rng(P)
    feat = torch.from_numpy((2e17 * np.clip(rng.normal(size=(3, P)), -4.9, 4.9)).astype(np.float32)).cuda()
    out, mean, rstd = rk.rocket_layer_norm(feat)
    _check_forward(feat, None, None, EPS, out, mean, rstd)
