"""Layers around the whitening, host side: the oracle's gradients against differences, workspace sizes, refusals (no kernel runs)."""
import numpy as np
import pytest

from oracle import layer_oracle as lo
from paper_2010_01546_amd import binding as b

FAKE = 0x10000   # aligned, never dereferenced: validation fails first


def differences(f, x, h=1e-6):
    """Central differences of the scalar f over the entries of x; error about h^2 |f'''| + 1e-16 |f| / h."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        x[i] = keep
    return g


def test_oracle_norm_gradient_against_differences():
    rng = np.random.default_rng(3)
    h, w, c, dh = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    f = lambda: float(np.sum(c * lo.rms_norm(h, w, 1e-3)) + np.sum(dh * h))  # noqa: E731
    dx, dw = lo.rms_norm_grad(h, w, 1e-3, c, dh)
    assert np.allclose(differences(f, h), dx, atol=1e-7)
    assert np.allclose(differences(f, w), dw, atol=1e-7)


@pytest.mark.parametrize("kind", lo.ACTS)
def test_oracle_gated_gradient_against_differences(kind):
    rng = np.random.default_rng(4)
    X, Wg, Wu, bg, bu, c = (rng.standard_normal(s) for s in ((5, 4), (3, 4), (3, 4), (3,), (3,), (5, 3)))
    f = lambda: float(np.sum(c * lo.gated(X, Wg, Wu, kind, bg, bu)))  # noqa: E731
    got = lo.gated_grad(X, Wg, Wu, kind, c, bg, bu)
    for x, g in zip((X, Wg, Wu, bg, bu), got):
        assert np.allclose(differences(f, x), g, atol=1e-7)
    # the centred gradient of W (x - mu) + b: the plain one of the same outputs, with the mean taken out of the rows
    mu = X.mean(0)
    cen = lo.gated_grad(X - mu, Wg, Wu, kind, c, bg + Wg @ mu, bu + Wu @ mu)
    for a, g in zip(lo.gated_grad(X, Wg, Wu, kind, c, bg, bu, mu=mu), cen):
        assert np.allclose(a, g, atol=1e-12)


def test_oracle_quantisation():
    q, s = lo.int8_steps(np.array([[1.0, -2.0, 0.0], [0.0, 0.0, 0.0]]))
    assert np.allclose(q, [[63.5, -127, 0], [0, 0, 0]]) and np.allclose(s, [2 / 127, 0])


def test_workspace_sizes():
    d = b.conv_desc(100, 64)
    assert b.fw_workspace_bytes(b.FW_OP_RMS_NORM_GRAD, 64, 0, d) >= 64 * 4
    for op in (b.FW_OP_GATED_GRAD, b.FW_OP_RMS_NORM_GRAD):
        assert b.fw_workspace_bytes(op, 64, 32, d) > 0
        assert b.fw_workspace_bytes(op, 64, 32, d, b.FW_BF16) % 256 == 0
    for op in (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD, b.FW_OP_INT8_PRODUCT, b.FW_OP_RMS_NORM_GRAD):
        assert b.fw_workspace_bytes(op, 64, 32, None) == 0          # no rows given
        assert b.fw_workspace_bytes(op, 32769, 32, b.conv_desc(8, 32769)) == 0
        assert b.fw_workspace_bytes(op, 0, 32, d) == 0
    assert b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, 64, 65537, d) == 0


def statuses(call, good, changes):
    for change, want in changes:
        args = dict(good, **change)
        assert call(*args.values()) == want, (change, want)


def test_norm_refusals():
    L, I, U, A, W = b.lib, b.FW_ERR_INVALID_ARG, b.FW_ERR_UNSUPPORTED, b.FW_ERR_ALIGNMENT, b.FW_ERR_WORKSPACE
    p = lambda k: FAKE + 4096 * k  # noqa: E731
    good = dict(X=p(1), R=p(2), dt=0, N=4, M=8, w=p(3), eps=1e-5, H=p(4), Y=p(5), q=p(6), qs=p(7), stream=None)
    statuses(L.fw_rms_norm, good, [
        (dict(X=None), I), (dict(Y=None, q=None, qs=None), I), (dict(q=None), I), (dict(qs=None), I), (dict(eps=0.0), I), (dict(eps=-1.0), I),
        (dict(eps=float("nan")), I), (dict(N=0), I), (dict(N=-3), I), (dict(M=0), I), (dict(dt=2), I), (dict(Y=p(1)), I), (dict(Y=p(2)), I),
        (dict(Y=p(4)), I), (dict(q=p(1)), I), (dict(q=p(4)), I), (dict(q=p(5)), I), (dict(M=32769), U), (dict(N=(1 << 21) + 1), U), (dict(X=p(1) + 8), A), (dict(qs=p(7) + 4), A), (dict(w=p(3) + 4), A)])
    good = dict(H=p(1), dt=1, N=4, M=8, w=p(3), eps=1e-5, dY=p(2), dH=p(4), dX=p(5), dw=p(6), ws=p(7), n=1 << 20, stream=None)
    statuses(L.fw_rms_norm_grad, good, [
        (dict(H=None), I), (dict(dY=None), I), (dict(dX=None, dw=None), I), (dict(eps=0.0), I), (dict(dX=p(1)), I), (dict(N=0), I), (dict(dt=-1), I),
        (dict(M=40000), U), (dict(dX=p(5) + 2), A), (dict(ws=None), W), (dict(n=16), W)])
    good = dict(X=p(1), dt=0, N=4, M=8, q=p(2), qs=p(3), stream=None)
    statuses(L.fw_int8_rows, good, [
        (dict(X=None), I), (dict(q=None), I), (dict(qs=None), I), (dict(q=p(1)), I), (dict(N=0), I), (dict(M=-1), I), (dict(dt=3), I), (dict(M=32769), U),
        (dict(q=p(2) + 1), A)])


def test_gated_refusals():
    L, I, U, A, W = b.lib, b.FW_ERR_INVALID_ARG, b.FW_ERR_UNSUPPORTED, b.FW_ERR_ALIGNMENT, b.FW_ERR_WORKSPACE
    p = lambda k: FAKE + 4096 * k  # noqa: E731
    good = dict(X=p(1), dt=0, N=4, M=8, S=6, Wg=p(2), Wu=p(3), bg=None, bu=None, act=0, H=p(4), Z=p(5), ws=p(6), n=1 << 20, stream=None)
    statuses(L.fw_gated_forward, good, [
        (dict(X=None), I), (dict(Wg=None), I), (dict(Wu=None), I), (dict(H=None), I), (dict(act=4), I), (dict(act=-1), I), (dict(dt=5), I), (dict(N=0), I),
        (dict(M=0), I), (dict(S=0), I), (dict(H=p(1)), I), (dict(Z=p(4)), I), (dict(Z=p(1)), I), (dict(M=32769), U), (dict(S=65537), U),
        (dict(Wu=p(3) + 2), A), (dict(bg=p(7) + 4), A), (dict(Z=p(5) + 8), A)])
    assert b.fw_workspace_bytes(b.FW_OP_GATED_FORWARD, 8, 6, b.conv_desc(100, 8)) > 0
    statuses(L.fw_gated_forward, good, [(dict(N=100, ws=None), W), (dict(N=100, n=0), W)])
    good = dict(X=p(1), dt=1, N=4, M=8, S=6, Wg=p(2), Wu=p(3), Z=p(4), dH=p(5), mu=None, dX=p(6), dWg=p(7), dWu=p(8), dbg=p(9), dbu=p(10), ws=p(11),
                n=1 << 20, stream=None)
    statuses(L.fw_gated_grad, good, [
        (dict(X=None), I), (dict(Wg=None), I), (dict(Wu=None), I), (dict(Z=None), I), (dict(dH=None), I), (dict(dWg=None), I), (dict(dWu=None), I),
        (dict(dbg=None), I), (dict(dbu=None), I), (dict(dX=None, dWg=None, dWu=None, dbg=None, dbu=None), I), (dict(dX=p(1)), I), (dict(dX=p(5)), I),
        (dict(dX=p(4)), I), (dict(dWg=p(8)), I), (dict(dWg=p(2)), I), (dict(dWu=p(2)), I), (dict(dWu=p(1)), I), (dict(dX=p(7)), I), (dict(dX=p(2)), I),
        (dict(dWg=p(5)), I), (dict(dWu=p(5)), I), (dict(dWg=p(4)), I), (dict(dWu=p(4)), I), (dict(dbu=p(9)), I), (dict(dt=2), I), (dict(N=0), I),
        (dict(S=0), I), (dict(M=40000), U), (dict(S=70000), U), (dict(mu=p(12) + 4), A), (dict(dX=p(6) + 2), A), (dict(ws=None), W), (dict(n=64), W)])


def test_int8_refusals():
    L, I, U, A = b.lib, b.FW_ERR_INVALID_ARG, b.FW_ERR_UNSUPPORTED, b.FW_ERR_ALIGNMENT
    p = lambda k: FAKE + 4096 * k  # noqa: E731
    good = dict(Xq=p(1), sx=p(2), N=4, M=8, S=6, Wq=p(3), sw=p(4), b=None, Y=p(5), dt=0, ws=p(6), n=1 << 20, stream=None)
    statuses(L.fw_int8_product, good, [
        (dict(Xq=None), I), (dict(sx=None), I), (dict(Wq=None), I), (dict(sw=None), I), (dict(Y=None), I), (dict(Y=p(1)), I), (dict(Y=p(3)), I),
        (dict(N=0), I), (dict(M=0), I), (dict(S=0), I), (dict(dt=2), I), (dict(M=32769), U), (dict(S=65537), U), (dict(Xq=p(1) + 1), A),
        (dict(sw=p(4) + 4), A), (dict(ws=p(6) + 4), A)])
