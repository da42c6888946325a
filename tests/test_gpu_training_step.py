"""One training step as a program puts it together: soft transform, layer norm of the features, a linear head and a squared
loss, the backward passes, clipping, an update of every parameter.  Each piece's gradient has its own tests; here the loss's
gradient with respect to every parameter, through all of them, is compared with the oracle's convolutions and the formulas in
64 bits, and the step is run again with the updated kernels."""
import copy

import numpy as np
import pytest

import oracle
import paper_2301_08527_b200 as rk
from rocket_inputs import ar1_spike_series, generate_kernels

import parity as P

pytestmark = pytest.mark.gpu

LAM, SHIFT, EPS, MAX_NORM = 4.0, 0.0, 1e-5, 0.05
U = 2.0 ** -24


def _step(p, X, t, gamma, beta, w, half):
    import torch
    feat, arg = rk.rocket_transform_soft(p, X, LAM, SHIFT)
    y, mean, rstd = rk.rocket_layer_norm(feat, gamma, beta, EPS, out_dtype=torch.bfloat16 if half else None)
    res = y.float() @ w - t
    dout = 2.0 * res / res.numel()
    dw = y.float().t() @ dout
    dy = (dout[:, None] * w[None, :]).to(y.dtype)
    dfeat, dgamma, dbeta = rk.rocket_layer_norm_backward(dy, feat, mean, rstd, gamma)
    dW, db = rk.rocket_transform_soft_backward(p, X, LAM, SHIFT, dfeat, arg)
    grads = [dW, db, dgamma, dbeta, dw]
    raw = [g.clone() for g in grads]
    norm, _ = rk.rocket_clip_grad_norm(grads, MAX_NORM)
    return feat, arg, y, dy, raw, norm, grads


@pytest.mark.parametrize("half", [False, True])
def test_a_training_step_against_the_formulas(half):
    import torch
    C, L, K, N = 3, 400, 60, 10
    kp = generate_kernels(71, K, C, L)
    X = ar1_spike_series(72, N, C, L)
    rng = np.random.default_rng(73)
    t = rng.normal(size=N).astype(np.float32)
    gamma, beta = (1 + 0.2 * rng.normal(size=2 * K)).astype(np.float32), (0.1 * rng.normal(size=2 * K)).astype(np.float32)
    w = (rng.normal(size=2 * K) / np.sqrt(2 * K)).astype(np.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    p = rk.RocketParams.from_kernel_params(kp)
    params = [kp.weights.copy(), kp.bias.copy(), gamma, beta, w]
    for _ in range(2):
        feat, arg, y, dy, raw, norm, clipped = _step(p, dev(X), dev(t), dev(params[2]), dev(params[3]), dev(params[4]), half)
        kq = copy.copy(kp)
        kq.weights, kq.bias = params[0], params[1]
        f = feat.cpu().numpy()
        ref = oracle.forward(kq, X, lam=LAM, shift=SHIFT)
        soft, mx = P.split_features(f)
        P.check_soft_ppv(soft, ref)
        P.check_max(mx, ref)
        g64, b64, w64 = (a.astype(np.float64) for a in params[2:])
        f = f.astype(np.float64)
        m = f.mean(1, keepdims=True)
        r = 1 / np.sqrt(((f - m) ** 2).mean(1, keepdims=True) + EPS)
        xh = (f - m) * r
        # half a step of y's and dy's type, and the fp32 work before it: 200 units of 2^-24 of the terms' magnitudes (the
        # layer norm's own bound; the head's product of 120 terms in fp32)
        h = torch.finfo(y.dtype).eps / 2
        y64, dy64 = y.double().cpu().numpy(), dy.double().cpu().numpy()
        want_y = xh * g64 + b64
        assert np.all(np.abs(y64 - want_y) <= h * np.abs(want_y) + 200 * U * (np.abs(xh * g64) + np.abs(g64) + np.abs(b64)) + 1e-30)
        dout = 2 * (y64 @ w64 - t) / N
        size = 2 * (np.abs(y64) @ np.abs(w64) + np.abs(t)) / N
        want_dy = dout[:, None] * w64
        assert np.all(np.abs(dy64 - want_dy) <= h * np.abs(want_dy) + 200 * U * size[:, None] * np.abs(w64) + 1e-30)
        # from here on the pieces are given the rounded y and dy that the device was given
        u = dy64 * g64
        dfeat = r * (u - u.mean(1, keepdims=True) - xh * (u * xh).mean(1, keepdims=True))
        rW, rb = oracle.backward(kq, X, dfeat.astype(np.float32), arg.cpu().numpy(), lam=LAM, shift=SHIFT)
        P.check_grads(raw[0].cpu().numpy(), raw[1].cpu().numpy(), rW, rb)
        terms = [dy64[:, :, None] * xh[:, :, None], dy64[:, :, None], y64[:, :, None] * dout[:, None, None]]
        for got, term in zip(raw[2:], terms):
            got, ref = got.cpu().numpy().astype(np.float64), term.sum(0)[:, 0]
            slack = 300 * U * np.abs(term).sum(0)[:, 0]
            if term is terms[2]:
                slack = slack + 200 * U * (np.abs(y64) * size[:, None]).sum(0)
            assert np.all(np.abs(got - ref) <= slack + 1e-30)
        total = sum(float((g.double() ** 2).sum()) for g in raw)
        assert abs(float(norm) - total ** 0.5) <= 2.0 ** -23 * total ** 0.5
        c = min(1.0, MAX_NORM / (total ** 0.5 + 1e-6))
        assert c < 1.0
        for a, b in zip(raw, clipped):
            assert np.allclose(b.cpu().numpy(), a.cpu().numpy().astype(np.float64) * c, rtol=6 * U, atol=2.0 ** -149)
        params = [a.astype(np.float32) - np.float32(0.1) * g.cpu().numpy() for a, g in zip(params, clipped)]
        p.set_weights(params[0], params[1])
    p.close()
