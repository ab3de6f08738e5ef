"""GPU parity of the layers around the whitening (norm, gated block, 8-bit product) against the float64 oracle.

Tolerances: U32 = 2^-24 and half(t) (2^-8 for bfloat16, 2^-24 for float32) are the most a rounding is off by, relative to its value; a
float32 sum of K terms in any order is off by at most (K + a few) U32 times the sum of the terms' magnitudes."""
import numpy as np
import pytest
import torch

import workloads as wl
from gpu_common import DEV, b, dev, relF, workspace
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
FDT = {"f32": b.FW_F32, "bf16": b.FW_BF16}
EPS = 1e-5


def rows(rng, n, m, dtype, scale=1.0):
    x = (scale * rng.standard_normal((n, m)) * np.exp(0.5 * rng.standard_normal(m))).astype(np.float32)
    return wl.round_to_bf16(x) if dtype == "bf16" else x


class Out:
    """An output with a guard behind it that no call may touch."""
    GUARD = 96

    def __init__(self, *shape, dtype):
        n = int(np.prod(shape))
        self.fill = 77 if dtype == torch.int8 else float("nan")
        self.buf = torch.full((n + self.GUARD,), self.fill, dtype=dtype, device=DEV)
        self.t = self.buf[:n].view(*shape)

    def host(self):
        tail = self.buf[self.t.numel():].float()
        assert bool((tail == 77).all() if self.fill == 77 else torch.isnan(tail).all()), "written behind the end"
        return self.t.float().cpu().numpy().astype(np.float64)


def within(got, want, tol, what=""):
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, first at {i}: {got[i]!r} for {want[i]!r}, allowed {np.broadcast_to(tol, got.shape)[i]:.3g}")


# ---------------------------------------------------------------------------------------------------------------- norm

NORM_SIZES = [(1, 1), (1, 7), (2, 8), (3, 64), (5, 129), (4, 512), (7, 513), (3, 1025), (6, 2048), (2, 2049), (1, 4608), (3, 8192), (2, 8197),
              (2, 16384), (1, 16391), (2, 32768), (65, 48), (1030, 72), (4101, 33), (9, 9), (17, 507), (11, 2043), (9, 6139), (3, 16381), (3, 32763), (1035, 2307), (2, 16393), (2, 24577), (3, 24576), (2, 12285), (3, 12289)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M", NORM_SIZES)
def test_norm(N, M, dtype):
    rng = np.random.default_rng(N * 100003 + M)
    t, dt = TDT[dtype], FDT[dtype]
    X, R = rows(rng, N, M, dtype), rows(rng, N, M, dtype, 2.0)
    w = (1 + 0.2 * rng.standard_normal(M)).astype(np.float32)
    Xd, Rd = dev(X, t), dev(R, t)
    H, Y, q, qs = Out(N, M, dtype=t), Out(N, M, dtype=t), Out(N, M, dtype=torch.int8), Out(N, dtype=torch.float32)
    b.fw_rms_norm(Xd, Rd, dt, N, M, dev(w), EPS, H.t, Y.t, q.t, qs.t)
    torch.cuda.synchronize()
    held = (Xd.float() + Rd.float()).to(t)
    assert torch.equal(H.t, held)
    h = held.float().cpu().numpy().astype(np.float64)
    want = lo.rms_norm(h, w, EPS)
    within(Y.host(), want, np.abs(want) * (HALF[dtype] + 4 * U32), "Y")          # rho, two products, the last rounding
    steps, s = lo.int8_steps(want)
    within(q.host(), steps, 0.5 + 1e-9, "q")
    within(qs.host(), s, s * 1.01 * U32, "qs")
    # without the residual, without w, 8 bits alone and 16 or 32 bits alone: each its own call
    Y2, q2, qs2 = Out(N, M, dtype=t), Out(N, M, dtype=torch.int8), Out(N, dtype=torch.float32)
    b.fw_rms_norm(held, None, dt, N, M, None, EPS, None, Y2.t)
    b.fw_rms_norm(held, None, dt, N, M, dev(w), EPS, None, None, q2.t, qs2.t)
    torch.cuda.synchronize()
    want = lo.rms_norm(h, None, EPS)
    within(Y2.host(), want, np.abs(want) * (HALF[dtype] + 4 * U32), "Y without w")
    assert torch.equal(q2.t, q.t) and torch.equal(qs2.t, qs.t)
    q2.host(), qs2.host()
    # the sum in place of either addend
    X2, R2 = Xd.clone(), Rd.clone()
    b.fw_rms_norm(X2, Rd, dt, N, M, dev(w), EPS, X2, Y2.t)
    torch.cuda.synchronize()
    assert torch.equal(X2, held) and torch.equal(Y2.t, Y.t)
    b.fw_rms_norm(Xd, R2, dt, N, M, dev(w), EPS, R2, Y2.t)
    torch.cuda.synchronize()
    assert torch.equal(R2, held) and torch.equal(Y2.t, Y.t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M", NORM_SIZES)
def test_norm_gradient(N, M, dtype):
    rng = np.random.default_rng(N * 100019 + M)
    t, dt = TDT[dtype], FDT[dtype]
    Hh, dY, dHh = rows(rng, N, M, dtype), rows(rng, N, M, dtype, 0.1), rows(rng, N, M, dtype, 0.1)
    w = (1 + 0.2 * rng.standard_normal(M)).astype(np.float32)
    Hd, dYd, dHd, wd = dev(Hh, t), dev(dY, t), dev(dHh, t), dev(w)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_RMS_NORM_GRAD, M, 0, b.conv_desc(N, M), dt))
    dX, dw = Out(N, M, dtype=t), Out(M, dtype=torch.float32)
    b.fw_rms_norm_grad(Hd, dt, N, M, wd, EPS, dYd, dHd, dX.t, dw.t, ws)
    torch.cuda.synchronize()
    want, want_w = lo.rms_norm_grad(Hh, w, EPS, dY, dHh)
    rho = 1 / np.sqrt(np.mean(lo.f64(Hh) ** 2, axis=1, keepdims=True) + EPS)
    first = np.abs(rho * lo.f64(dY) * w)
    second = np.abs(Hh * rho ** 3 * np.mean(lo.f64(dY) * w * Hh, axis=1, keepdims=True))
    within(dX.host(), want, np.abs(want) * HALF[dtype] + 5 * U32 * (first + second + np.abs(dHh)), "dX")
    terms = np.abs(lo.f64(dY) * Hh * rho)
    within(dw.host(), want_w, (min(N, 100 + N // 1024) + 4) * U32 * terms.sum(0), "dw")   # chains: a workgroup's rows, a slice, the slices
    # one output at a time, no residual path, no w, in place of dY and of dH
    dX2, dw2 = Out(N, M, dtype=t), Out(M, dtype=torch.float32)
    b.fw_rms_norm_grad(Hd, dt, N, M, wd, EPS, dYd, dHd, dX2.t, None)
    b.fw_rms_norm_grad(Hd, dt, N, M, wd, EPS, dYd, None, None, dw2.t, ws)
    torch.cuda.synchronize()
    assert torch.equal(dX2.t, dX.t) and torch.equal(dw2.t, dw.t)
    for src in ("dY", "dH"):
        a, c = dYd.clone(), dHd.clone()
        b.fw_rms_norm_grad(Hd, dt, N, M, wd, EPS, a, c, a if src == "dY" else c, dw2.t, ws)
        torch.cuda.synchronize()
        assert torch.equal(a if src == "dY" else c, dX.t) and torch.equal(dw2.t, dw.t)
    b.fw_rms_norm_grad(Hd, dt, N, M, None, EPS, dYd, None, dX2.t, None)
    torch.cuda.synchronize()
    want = lo.rms_norm_grad(Hh, None, EPS, dY)[0]
    first, second = np.abs(rho * lo.f64(dY)), np.abs(Hh * rho ** 3 * np.mean(lo.f64(dY) * Hh, axis=1, keepdims=True))
    within(dX2.host(), want, np.abs(want) * HALF[dtype] + 5 * U32 * (first + second), "dX without w")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_extreme_rows(dtype):
    t, dt, M = TDT[dtype], FDT[dtype], 70
    X = np.ones((8, M), dtype=np.float32)
    X[0] = 0.0
    X[1] *= 1e30             # squares beyond float32
    X[2] *= 1e-30
    X[3, 5] = np.inf
    X[4, 69] = np.nan
    X[5, :] = -3.0
    X[6, 1:] = 0.0
    X[7, 0] = 250.0
    X = wl.round_to_bf16(X) if dtype == "bf16" else X
    Y, q, qs = Out(8, M, dtype=t), Out(8, M, dtype=torch.int8), Out(8, dtype=torch.float32)
    b.fw_rms_norm(dev(X, t), None, dt, 8, M, None, EPS, None, Y.t, q.t, qs.t)
    q3, qs3 = Out(8, M, dtype=torch.int8), Out(8, dtype=torch.float32)
    b.fw_int8_rows(dev(X, t), dt, 8, M, q3.t, qs3.t)
    torch.cuda.synchronize()
    fine = [0, 1, 2, 5, 6, 7]
    want = lo.rms_norm(X[fine], None, EPS)
    within(Y.host()[fine], want, np.abs(want) * (HALF[dtype] + 4 * U32))
    for got, scale, src in ((q.host(), qs.host(), want), (q3.host(), qs3.host(), lo.f64(X[fine]))):
        steps, s = lo.int8_steps(src)
        within(got[fine], steps, 0.5 + 1e-9)
        within(scale[fine], s, s * 1.01 * U32)
        assert scale[0] == 0 and np.isnan(scale[[3, 4]]).all() and not got[[0, 3, 4]].any()
    assert np.isnan(Y.host()[3, 5]) and np.isnan(Y.host()[4]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M", [(1, 1), (3, 9), (17, 64), (5, 1000), (2, 2305), (1, 12288), (2, 32768), (300, 576)])
def test_int8_rows(N, M, dtype):
    rng = np.random.default_rng(N + M)
    X = rows(rng, N, M, dtype)
    q, qs = Out(N, M, dtype=torch.int8), Out(N, dtype=torch.float32)
    b.fw_int8_rows(dev(X, TDT[dtype]), FDT[dtype], N, M, q.t, qs.t)
    torch.cuda.synchronize()
    steps, s = lo.int8_steps(X)
    within(q.host(), steps, 0.5 + 1e-9)
    within(qs.host(), s, s * 1.01 * U32)
    assert np.abs(q.host()).max() == 127


# --------------------------------------------------------------------------------------------------------- gated block

GATED_SIZES = [(1, 1, 1), (1, 8, 5), (1, 64, 128), (2, 33, 65), (3, 130, 64), (7, 256, 200), (16, 576, 96), (17, 72, 257), (31, 1000, 33),
               (32, 512, 512), (33, 40, 130), (64, 64, 64), (65, 96, 129), (127, 129, 513), (128, 576, 256), (130, 200, 1000), (200, 1153, 67),
               (257, 320, 384), (300, 72, 700), (513, 257, 300), (1100, 64, 72), (1, 2304, 300), (4, 4608, 40), (520, 513, 1030), (1, 3, 70), (18, 4, 33), (40, 1030, 1100), (64, 4099, 300), (64, 2001, 130), (9, 70, 4100)]
ACT = {k: i for i, k in enumerate(lo.ACTS)}


def act_of(N, M, S):
    return lo.ACTS[(N + M + S) % 4]


def gated_inputs(N, M, S, dtype, bias):
    rng = np.random.default_rng(N * 7919 + M * 31 + S)
    X = rows(rng, N, M, dtype)
    Wg, Wu = (rows(rng, S, M, dtype, M ** -0.5) for _ in range(2))
    bg, bu = ((0.3 * rng.standard_normal(S)).astype(np.float32) if bias else None for _ in range(2))
    return rng, X, Wg, Wu, bg, bu


def run_forward(X, Wg, Wu, bg, bu, kind, dtype, keep=True):
    (N, M), S, t = X.shape, Wg.shape[0], TDT[dtype]
    H, Z = Out(N, S, dtype=t), Out(2, N, S, dtype=torch.float32) if keep else None
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_FORWARD, M, S, b.conv_desc(N, M), FDT[dtype]))
    ws.fill_(255)
    b.fw_gated_forward(dev(X, t), FDT[dtype], N, M, S, dev(Wg, t), dev(Wu, t), None if bg is None else dev(bg), None if bu is None else dev(bu),
                       ACT[kind], H.t, Z.t if keep else None, ws)
    torch.cuda.synchronize()
    return H, Z


def check_forward(H, Z, X, Wg, Wu, bg, bu, kind, dtype):
    M = X.shape[1]
    g, u = lo.projections(X, Wg, Wu, bg, bu)
    mag = lambda W, c: np.abs(lo.f64(X)) @ np.abs(lo.f64(W)).T + (0 if c is None else np.abs(c))  # noqa: E731
    eg, eu = (M + 8) * U32 * mag(Wg, bg), (M + 8) * U32 * mag(Wu, bu)
    a, da = lo.act(kind, g), lo.act_slope(kind, g)
    # |act'| <= 1.13 for all of them, act evaluated to a few units of float32 of max(|g|, 1)
    tol = 1.2 * eg * (np.abs(u) + eu) + np.abs(a) * eu + 16 * U32 * np.abs(g * u)
    within(H, a * u, tol + np.abs(a * u) * HALF[dtype] + 1e-38, "H")
    if Z is None:
        return
    # |act''| <= 1.2; the slope of relu is that of a g on the same side of zero
    sure = np.abs(g) > eg if kind == "relu" else np.ones_like(g, dtype=bool)
    tol = np.abs(u) * 1.2 * eg + 1.2 * eu + 16 * U32 * (1 + np.abs(g)) * np.abs(u)
    within(np.where(sure, Z[0], 0), np.where(sure, u * da, 0), tol + 1e-38, "Z[0]")
    within(Z[1], a, 1.2 * eg + 16 * U32 * np.abs(g) + 1e-38, "Z[1]")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", GATED_SIZES)
def test_gated_forward(N, M, S, dtype):
    kind, bias = act_of(N, M, S), (N + S) % 3 != 0
    _, X, Wg, Wu, bg, bu = gated_inputs(N, M, S, dtype, bias)
    H, Z = run_forward(X, Wg, Wu, bg, bu, kind, dtype)
    check_forward(H.host(), Z.host(), X, Wg, Wu, bg, bu, kind, dtype)
    H2, _ = run_forward(X, Wg, Wu, bg, bu, kind, dtype, keep=False)
    assert torch.equal(H2.t, H.t)
    H2.host()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", lo.ACTS)
@pytest.mark.parametrize("N", [1, 70])
def test_gated_activations(N, kind, dtype):
    _, X, Wg, Wu, bg, _ = gated_inputs(N, 72, 100, dtype, True)
    H, Z = run_forward(4 * X, Wg, Wu, bg, None, kind, dtype)
    check_forward(H.host(), Z.host(), 4 * X, Wg, Wu, bg, None, kind, dtype)


def two_numbers(N, S):
    """bfloat16: dg and du are held as two bfloat16 numbers each."""
    return N * S <= 1 << 19


def rounded_product(a, c, dtype):
    """dH times a factor as the block's gradient has it: in float32, then rounded to the type (large bfloat16 blocks)."""
    p = (lo.f64(a) * c).astype(np.float32)
    return lo.f64(wl.round_to_bf16(p) if dtype == "bf16" and not two_numbers(*a.shape) else p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", GATED_SIZES)
def test_gated_gradient(N, M, S, dtype):
    kind, bias, t, dt = act_of(N, M, S), (N + S) % 3 != 0, TDT[dtype], FDT[dtype]
    rng, X, Wg, Wu, bg, bu = gated_inputs(N, M, S, dtype, bias)
    dH = rows(rng, N, S, dtype, 0.1)
    mu = lo.f64(X).mean(0).astype(np.float32) + 0.1 if (N + M) % 2 else None
    _, Z = run_forward(X, Wg, Wu, bg, bu, kind, dtype)
    Zh = Z.host()
    dX, dWg, dWu, dbg, dbu = Out(N, M, dtype=t), Out(S, M, dtype=t), Out(S, M, dtype=t), Out(S, dtype=t), Out(S, dtype=t)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    ws.fill_(255)                                                  # NaN in every type: nothing may be read before it is written
    Xd, Wgd, Wud, dHd, mud = dev(X, t), dev(Wg, t), dev(Wu, t), dev(dH, t), None if mu is None else dev(mu)
    b.fw_gated_grad(Xd, dt, N, M, S, Wgd, Wud, Z.t, dHd, mud, dX.t, dWg.t, dWu.t, dbg.t, dbu.t, ws)
    torch.cuda.synchronize()
    dg, du = rounded_product(dH, Zh[0], dtype), rounded_product(dH, Zh[1], dtype)
    half = HALF[dtype]
    want = lo.gated_grad_from(dg, du, X, Wg, Wu, mu)
    ag, au, aX = np.abs(dg), np.abs(du), np.abs(lo.f64(X)) + (0 if mu is None else np.abs(mu))
    # what is left of dg and du: a float32 rounding; of two bfloat16 numbers the second's, half a step (2^-8) of what the first left (2^-8)
    more = U32 if dtype == "f32" else U32 + 2.0 ** -16 if two_numbers(N, S) else 0.0
    within(dX.host(), want[0], ((2 * S + 8) * U32 + more) * (ag @ np.abs(lo.f64(Wg)) + au @ np.abs(lo.f64(Wu))) + half * np.abs(want[0]), "dX")
    within(dWg.host(), want[1], ((2 * N + 8) * U32 + more) * (ag.T @ aX) + half * np.abs(want[1]), "dWg")
    within(dWu.host(), want[2], ((2 * N + 8) * U32 + more) * (au.T @ aX) + half * np.abs(want[2]), "dWu")
    for got, factor, what in ((dbg, Zh[0], "dbg"), (dbu, Zh[1], "dbu")):      # of the products before their rounding to the type
        d = lo.f64(dH) * factor
        within(got.host(), d.sum(0), (N + 5) * U32 * np.abs(d).sum(0) + half * np.abs(d.sum(0)), what)
    # against the whole formula in 64 bits: dg and du (large blocks) and the results have a rounding each, of at most `half`; float32 adds
    # its sums
    full = lo.gated_grad(X, Wg, Wu, kind, dH, bg, bu, mu)
    if kind != "relu":
        for got, w, what in zip((dX, dWg, dWu), full, ("dX", "dWg", "dWu")):
            assert relF(got.host(), w) < (2 * half + 1e-4 if dtype == "bf16" else 2e-5), what
    # one group of outputs at a time
    alone = [Out(N, M, dtype=t), Out(S, M, dtype=t), Out(S, M, dtype=t), Out(S, dtype=t), Out(S, dtype=t)]
    b.fw_gated_grad(Xd, dt, N, M, S, Wgd, Wud, Z.t, dHd, None, alone[0].t, None, None, None, None, ws)
    b.fw_gated_grad(Xd, dt, N, M, S, Wgd, Wud, Z.t, dHd, mud, None, alone[1].t, alone[2].t, None, None, ws)
    b.fw_gated_grad(Xd, dt, N, M, S, Wgd, Wud, Z.t, dHd, None, None, None, None, alone[3].t, alone[4].t, ws)
    torch.cuda.synchronize()
    for a, c in zip(alone, (dX, dWg, dWu, dbg, dbu)):
        assert torch.equal(a.t, c.t)
        a.host()


# few rows, where each workgroup has its columns' whole sums, and a few more: row ends of every kind, few and many columns
FEW_SIZES = [(1, 7, 3), (2, 8, 259), (4, 33, 1), (15, 129, 300), (16, 577, 1030), (17, 1100, 33), (31, 136, 4100), (32, 2305, 6145), (3, 64, 8200),
             (1, 12289, 20), (50, 129, 300), (64, 1000, 270), (40, 2305, 4200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", FEW_SIZES + [(49, 127, 517), (64, 1000, 30)])
def test_gated_few_rows(N, M, S, dtype):
    kind = act_of(N, M, S)
    _, X, Wg, Wu, bg, bu = gated_inputs(N, M, S, dtype, S % 2 == 0)
    H, Z = run_forward(X, Wg, Wu, bg, bu, kind, dtype)
    check_forward(H.host(), Z.host(), X, Wg, Wu, bg, bu, kind, dtype)
    # the last weights of a row in front of entries that are no part of it: an infinite row of the weights reaches its own column alone
    Wg[0] = np.inf
    H2, _ = run_forward(X, Wg, Wu, bg, bu, kind, dtype, keep=False)
    assert torch.equal(H2.t[:, 1:], H.t[:, 1:])


@pytest.mark.parametrize("N,M,S", FEW_SIZES)
def test_int8_few_rows(N, M, S):
    rng = np.random.default_rng(N + 13 * M + 7 * S)
    Xq, Wq = rng.integers(-128, 128, (N, M)).astype(np.int8), rng.integers(-128, 128, (S, M)).astype(np.int8)
    Y, ones = Out(N, S, dtype=torch.float32), torch.ones(max(N, S), device=DEV)
    ws = b.fw_workspace_bytes(b.FW_OP_INT8_PRODUCT, M, S, b.conv_desc(N, M), b.FW_F32)
    b.fw_int8_product(dev(Xq, torch.int8), ones, N, M, S, dev(Wq, torch.int8), ones, None, Y.t, b.FW_F32, workspace(ws) if ws else None)
    torch.cuda.synchronize()
    want = Xq.astype(np.int64) @ Wq.astype(np.int64).T
    within(Y.host(), want.astype(np.float64), np.abs(want) * U32)


def test_norm_gradient_of_extreme_rows():
    """Rows whose rho^3 lies outside float32, on either side."""
    rng = np.random.default_rng(5)
    M, eps = 70, 1e-38
    H = (rng.standard_normal((3, M)) * np.array([[1e25], [1.0], [1e-16]])).astype(np.float32)
    dY = rng.standard_normal((3, M)).astype(np.float32)
    dX = Out(3, M, dtype=torch.float32)
    b.fw_rms_norm_grad(dev(H), b.FW_F32, 3, M, None, eps, dev(dY), None, dX.t, None)
    torch.cuda.synchronize()
    eps = float(np.float32(eps))
    want = lo.rms_norm_grad(H, None, eps, dY)[0]
    rho = 1 / np.sqrt(np.mean(lo.f64(H) ** 2, axis=1, keepdims=True) + eps)
    first, second = np.abs(rho * dY), np.abs(H * rho ** 3 * np.mean(lo.f64(dY) * H, axis=1, keepdims=True))
    within(dX.host(), want, U32 * np.abs(want) + 5 * U32 * (first + second), "dX")


@pytest.mark.parametrize("kind", lo.ACTS)
def test_gated_with_extreme_gates(kind):
    """g as large as its type allows: the value is g or zero, the slope one or zero."""
    X = np.ones((2, 1), dtype=np.float32)
    Wg = wl.round_to_bf16(np.array([1e5, -1e5, 1e20, -1e20, 3e38, -3e38], dtype=np.float32)[:, None])
    Wu = np.full((6, 1), 0.5, dtype=np.float32)
    H, Z = run_forward(X, Wg, Wu, None, None, kind, "bf16")
    on = (Wg[:, 0] > 0).astype(np.float64)
    for n in range(2):
        within(Z.host()[0][n], 0.5 * on, 0.5 * on * 4 * U32, "Z[0]")
        within(Z.host()[1][n], np.where(on, lo.f64(Wg[:, 0]), 0.0), np.abs(Wg[:, 0]) * on * 4 * U32, "Z[1]")
        within(H.host()[n], np.where(on, 0.5 * lo.f64(Wg[:, 0]), 0.0), np.abs(Wg[:, 0]) * on * HALF["bf16"], "H")


# -------------------------------------------------------------------------------------------------------- 8-bit product

INT8_SIZES = [(1, 1, 1), (1, 16, 5), (1, 4608, 100), (2, 33, 65), (3, 130, 64), (7, 1000, 200), (16, 576, 96), (17, 72, 257), (32, 512, 512), (33, 48, 130),
              (64, 64, 64), (65, 97, 129), (128, 576, 256), (130, 208, 1000), (257, 320, 384), (513, 257, 300), (1100, 64, 72), (5, 32768, 9), (300, 1153, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", INT8_SIZES)
def test_int8_product(N, M, S, dtype):
    rng = np.random.default_rng(N + 13 * M + 7 * S)
    Xq = rng.integers(-128, 128, (N, M)).astype(np.int8)
    Wq = rng.integers(-128, 128, (S, M)).astype(np.int8)
    if N == 5:
        Xq[0], Wq[0], Wq[1] = -128, -128, 127                      # the largest sums there are
    sx, sw = (np.exp(rng.standard_normal(n)).astype(np.float32) * 1e-2 for n in (N, S))
    sx[0] = 0.0 if N > 2 and N != 5 else sx[0]
    bias = rng.standard_normal(S).astype(np.float32) if (N + S) % 2 else None
    Y = Out(N, S, dtype=TDT[dtype])
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_INT8_PRODUCT, M, S, b.conv_desc(N, M), FDT[dtype]))
    ws.fill_(255)
    b.fw_int8_product(dev(Xq, torch.int8), dev(sx), N, M, S, dev(Wq, torch.int8), dev(sw), None if bias is None else dev(bias), Y.t, FDT[dtype], ws)
    torch.cuda.synchronize()
    want = lo.int8_product(Xq, sx, Wq, sw, bias)
    plain = np.abs(lo.int8_product(Xq, sx, Wq, sw))
    within(Y.host(), want, 4 * U32 * (plain + (0 if bias is None else np.abs(bias))) + HALF[dtype] * np.abs(want))


@pytest.mark.parametrize("N,M,S", [(2100, 520, 4200), (2304, 192, 4608)])
def test_many_tiles(N, M, S):
    """More tiles than compute units: whole rounds of them, and a rest that is cut into runs; bfloat16 and 8 bits."""
    t, dt = torch.bfloat16, b.FW_BF16
    rng, X, Wg, Wu, bg, bu = gated_inputs(N, M, S, "bf16", True)
    H, Z = run_forward(X, Wg, Wu, bg, bu, "silu", "bf16")
    check_forward(H.host(), Z.host(), X, Wg, Wu, bg, bu, "silu", "bf16")
    dH, mu = rows(rng, N, S, "bf16", 0.1), lo.f64(X).mean(0).astype(np.float32)
    dX, dWg, dWu = Out(N, M, dtype=t), Out(S, M, dtype=t), Out(S, M, dtype=t)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    ws.fill_(255)
    b.fw_gated_grad(dev(X, t), dt, N, M, S, dev(Wg, t), dev(Wu, t), Z.t, dev(dH, t), dev(mu), dX.t, dWg.t, dWu.t, None, None, ws)
    torch.cuda.synchronize()
    Zh = Z.host()
    dg, du = rounded_product(dH, Zh[0], "bf16"), rounded_product(dH, Zh[1], "bf16")
    want, half = lo.gated_grad_from(dg, du, X, Wg, Wu, mu), HALF["bf16"]
    ag, au, aX = np.abs(dg), np.abs(du), np.abs(lo.f64(X)) + np.abs(mu)
    within(dX.host(), want[0], (2 * S + 8) * U32 * (ag @ np.abs(lo.f64(Wg)) + au @ np.abs(lo.f64(Wu))) + half * np.abs(want[0]), "dX")
    within(dWg.host(), want[1], (2 * N + 8) * U32 * (ag.T @ aX) + half * np.abs(want[1]), "dWg")
    within(dWu.host(), want[2], (2 * N + 8) * U32 * (au.T @ aX) + half * np.abs(want[2]), "dWu")
    Xq, Wq = rng.integers(-128, 128, (N, M)).astype(np.int8), rng.integers(-128, 128, (2 * S, M)).astype(np.int8)
    sx, sw, Y = np.full(N, 0.01, np.float32), np.full(2 * S, 0.02, np.float32), Out(N, 2 * S, dtype=torch.float32)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_INT8_PRODUCT, M, 2 * S, b.conv_desc(N, M)))
    b.fw_int8_product(dev(Xq, torch.int8), dev(sx), N, M, 2 * S, dev(Wq, torch.int8), dev(sw), None, Y.t, b.FW_F32, ws)
    torch.cuda.synchronize()
    want = lo.int8_product(Xq, sx, Wq, sw)
    within(Y.host(), want, 4 * U32 * np.abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", [(3, 70, 90), (70, 72, 100), (150, 129, 200)])
def test_gated_with_infinite_and_nan_entries(N, M, S, dtype):
    """They reach the results that the formula lets them reach, as the same infinities and NaN, and no others."""
    t, dt = TDT[dtype], FDT[dtype]
    rng, X, Wg, Wu, bg, bu = gated_inputs(N, M, S, dtype, True)
    X, Wg = X.copy(), Wg.copy()
    X[1, 5], X[2, M - 1] = np.inf, np.nan
    Wg[S - 1, 3] = -np.inf
    H, Z = run_forward(X, Wg, Wu, bg, bu, "relu", dtype)
    with np.errstate(all="ignore"):
        want = lo.gated(X, Wg, Wu, "relu", bg, bu)
    got = H.host()
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine)
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert fine[0, :S - 1].all() and not fine[1].all() and np.isnan(got[2]).all()
    assert relF(got[fine], want[fine]) < (2 * HALF["bf16"] if dtype == "bf16" else 1e-5)
    # gradient: finite factors, infinite entries of dH, X and the weights
    X[2, M - 1] = 0.5
    Zf = (0.3 + np.abs(rng.standard_normal((2, N, S)))).astype(np.float32)
    dH = rows(rng, N, S, dtype, 0.1)
    dH[0, 7], dH[2, 8] = np.inf, np.nan
    dX, dWg, dWu = Out(N, M, dtype=t), Out(S, M, dtype=t), Out(S, M, dtype=t)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    ws.fill_(255)
    b.fw_gated_grad(dev(X, t), dt, N, M, S, dev(Wg, t), dev(Wu, t), dev(Zf), dev(dH, t), None, dX.t, dWg.t, dWu.t, None, None, ws)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        dg, du = rounded_product(dH, lo.f64(Zf[0]), dtype), rounded_product(dH, lo.f64(Zf[1]), dtype)
        want = lo.gated_grad_from(dg, du, X, Wg, Wu)
    for got, w, what in zip((dX.host(), dWg.host(), dWu.host()), want, ("dX", "dWg", "dWu")):
        fine = np.isfinite(w)
        assert np.array_equal(np.isfinite(got), fine), what
        assert np.array_equal(got[np.isinf(w)], w[np.isinf(w)]), what
        assert fine.any() and relF(got[fine], w[fine]) < (2 * HALF["bf16"] if dtype == "bf16" else 1e-5), what


@pytest.mark.parametrize("N,M,S", [(150, 257, 300), (1000, 4608, 4000)])
def test_gated_of_nan(N, M, S):
    """float32, not a finite result: as the formula has it, and in a time like that of any other input."""
    t = lambda *shape: torch.full(shape, float("nan"), device=DEV)  # noqa: E731
    H, Z, dX, dWg, dWu = (Out(*shape, dtype=torch.float32) for shape in ((N, S), (2, N, S), (N, M), (S, M), (S, M)))
    X, W, dH = t(N, M), torch.ones(S, M, device=DEV), torch.ones(N, S, device=DEV)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_FORWARD, M, S, b.conv_desc(N, M)))
    b.fw_gated_forward(X, b.FW_F32, N, M, S, W, W, None, None, b.FW_ACT_SILU, H.t, Z.t, ws)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M)))
    b.fw_gated_grad(X, b.FW_F32, N, M, S, W, W, Z.t, dH, None, dX.t, dWg.t, dWu.t, None, None, ws)
    torch.cuda.synchronize()
    for x in (H, Z, dX, dWg, dWu):
        assert bool(torch.isnan(x.t).all())
    begin, end = torch.cuda.Event(True), torch.cuda.Event(True)
    begin.record()
    b.fw_gated_grad(X, b.FW_F32, N, M, S, W, W, Z.t, dH, None, dX.t, dWg.t, dWu.t, None, None, ws)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 100                           # ms; entry by entry it would be seconds


def test_offsets_beyond_32_bits():
    """Rows at the end of tensors of more than 2^31 entries."""
    t, dt = torch.bfloat16, b.FW_BF16
    gen = torch.Generator(device=DEV).manual_seed(1)
    N, M = 70000, 32768
    X = torch.randn(N, M, generator=gen, device=DEV, dtype=t)
    Y, q, qs = torch.empty_like(X), torch.empty(N, M, dtype=torch.int8, device=DEV), torch.empty(N, device=DEV)
    b.fw_rms_norm(X, None, dt, N, M, None, EPS, None, Y, q, qs)
    torch.cuda.synchronize()
    at = [0, 65535, N - 1]
    want = lo.rms_norm(X[at].float().cpu().numpy(), None, EPS)
    within(Y[at].float().cpu().numpy().astype(np.float64), want, np.abs(want) * (HALF["bf16"] + 4 * U32))
    within(q[at].cpu().numpy().astype(np.float64), lo.int8_steps(want)[0], 0.5 + 1e-9)
    del X, Y, q, qs
    N, M, S = 36000, 64, 65536
    X = torch.randn(N, M, generator=gen, device=DEV).to(t)
    Wg, Wu = ((torch.randn(S, M, generator=gen, device=DEV) / 8).to(t) for _ in range(2))
    H, Z, d = torch.empty(N, S, dtype=t, device=DEV), torch.empty(2, N, S, device=DEV), b.conv_desc(N, M)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_FORWARD, M, S, d, dt))
    b.fw_gated_forward(X, dt, N, M, S, Wg, Wu, None, None, b.FW_ACT_SILU, H, Z, ws)
    torch.cuda.synchronize()
    num = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
    for n in (0, N // 2, N - 1):
        check_forward(num(H[n:n + 1]), num(Z[:, n:n + 1]), num(X[n:n + 1]), num(Wg), num(Wu), None, None, "silu", "bf16")
    dH = H                                                            # any gradient will do
    dX, dWg, dWu = torch.empty_like(X), torch.empty_like(Wg), torch.empty_like(Wu)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, d, dt))
    b.fw_gated_grad(X, dt, N, M, S, Wg, Wu, Z, dH, None, dX, dWg, dWu, None, None, ws)
    torch.cuda.synchronize()
    n = N - 1
    D = [lo.f64((dH[n].float() * Z[k, n]).to(t).float().cpu().numpy()) for k in range(2)]
    want = D[0] @ num(Wg) + D[1] @ num(Wu)
    mag = np.abs(D[0]) @ np.abs(num(Wg)) + np.abs(D[1]) @ np.abs(num(Wu))
    within(num(dX[n]), want, (2 * S + 8) * U32 * mag + HALF["bf16"] * np.abs(want), "dX")
    s = [0, S // 2 + 1, S - 1]
    for k, got in ((0, dWg), (1, dWu)):
        D = num((dH[:, s].float() * Z[k][:, s]).to(t))
        want, mag = D.T @ num(X), np.abs(D).T @ np.abs(num(X))
        within(num(got[s]), want, (2 * N + 8) * U32 * mag + HALF["bf16"] * np.abs(want), "dW")


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, give what they give alone."""
    N, M, S, t, dt = 640, 512, 1536, torch.bfloat16, b.FW_BF16
    d, inputs = b.conv_desc(N, M), []
    for seed in (1, 2):
        rng = np.random.default_rng(seed)
        inputs.append([dev(rows(rng, *s, "bf16", 0.1), t) for s in ((N, M), (S, M), (S, M), (N, S))])

    def call(k, stream):
        X, Wg, Wu, dH = inputs[k]
        o = dict(H=torch.empty(N, S, dtype=t, device=DEV), Z=torch.empty(2, N, S, device=DEV), dX=torch.empty_like(X), dWg=torch.empty_like(Wg), dWu=torch.empty_like(Wu))
        w = [workspace(b.fw_workspace_bytes(op, M, S, d, dt)) for op in (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD)]
        torch.cuda.synchronize() if stream is None else None
        b.fw_gated_forward(X, dt, N, M, S, Wg, Wu, None, None, b.FW_ACT_SILU, o["H"], o["Z"], w[0], stream=stream)
        b.fw_gated_grad(X, dt, N, M, S, Wg, Wu, o["Z"], dH, None, o["dX"], o["dWg"], o["dWu"], None, None, w[1], stream=stream)
        return o, w

    alone = [call(k, None) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        both = [call(k, streams[k]) for k in range(2)]
        torch.cuda.synchronize()
        for k in range(2):
            for name in alone[k][0]:
                assert torch.equal(alone[k][0][name], both[k][0][name]), (turn, k, name)


# -------------------------------------------------------------------------------------------- as they are used together

def whitened_step(dtype, stream=None):
    """Residual and norm, gated block, its gradient with the centred rows, the norm's gradient; then the whitening's own calls on the
    block's input rows and weight gradients.  Returns host arrays of everything."""
    N, M, S, t, dt = 192, 64, 160, TDT[dtype], FDT[dtype]
    rng = np.random.default_rng(5)
    X, R = rows(rng, N, M, dtype) + 0.5, rows(rng, N, M, dtype)
    X = wl.round_to_bf16(X.astype(np.float32)) if dtype == "bf16" else X.astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal(M)).astype(np.float32)
    Wg, Wu = (rows(rng, S, M, dtype, M ** -0.5) for _ in range(2))
    dH, dStream = rows(rng, N, S, dtype, 0.1), rows(rng, N, M, dtype, 0.1)
    e = lambda *s, k=t: torch.empty(*s, dtype=k, device=DEV)  # noqa: E731
    d = b.conv_desc(N, M)
    wsf, wsg = (workspace(b.fw_workspace_bytes(op, M, S, d, dt)) for op in (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD))
    wsn = workspace(b.fw_workspace_bytes(b.FW_OP_RMS_NORM_GRAD, M, 0, d, dt))
    wsc = workspace(b.fw_workspace_bytes(b.FW_OP_COV_ACCUMULATE, M, 0, d, dt))
    wsd, wst = workspace(b.fw_workspace_bytes(b.FW_OP_COND_REDUCE_STEP, M)), workspace(b.fw_workspace_bytes(b.FW_OP_GRAD_TRANSFORM, M, S, None, dt))
    Xd, Rd, wd, Wgd, Wud, dHd, dSd = dev(X, t), dev(R, t), dev(w), dev(Wg, t), dev(Wu, t), dev(dH, t), dev(dStream, t)
    H, Y, A, Z, dY, dX, dw = e(N, M), e(N, M), e(N, S), e(2, N, S, k=torch.float32), e(N, M), e(N, M), e(M, k=torch.float32)
    dWg, dWu, Gg, Gu = e(S, M), e(S, M), e(S, M), e(S, M)
    f = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    C, s1, mu, Phi, phi, lbar = f(M, M), f(M), f(M), f(M, M), f(M), f(4)
    T, Q, Qs, Py, Psi, xi2, info = f(M, M), f(M, M), f(M, M), f(M, M), f(M, M), f(M), torch.zeros(8, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    b.fw_rms_norm(Xd, Rd, dt, N, M, wd, EPS, H, Y, stream=stream)
    b.fw_cov_accumulate(Y, dt, b.FW_LAYOUT_ROWS, d, C, s1, wsc, stream=stream)
    b.fw_cov_finalize(C, s1, N, M, 0.0, 1, mu, Phi, phi, lbar, stream=stream)
    st = b.cond_state(M, Phi, lbar, T, Q, Qs, Py, Psi, xi2)
    b.fw_cond_state_init(st, stream=stream)
    b.fw_cond_reduce_step(st, b.cond_params(), info, wsd, stream=stream)
    b.fw_gated_forward(Y, dt, N, M, S, Wgd, Wud, None, None, b.FW_ACT_SILU, A, Z, wsf, stream=stream)
    b.fw_gated_grad(Y, dt, N, M, S, Wgd, Wud, Z, dHd, mu, dY, dWg, dWu, None, None, wsg, stream=stream)
    b.fw_rms_norm_grad(H, dt, N, M, wd, EPS, dY, dSd, dX, dw, wsn, stream=stream)
    for G, out in ((dWg, Gg), (dWu, Gu)):
        b.fw_grad_transform(G, dt, S, M, None, Qs, out, wst, stream=stream)
    torch.cuda.synchronize()
    host = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
    got = {k: host(v) for k, v in dict(H=H, Y=Y, A=A, dY=dY, dX=dX, dw=dw, dWg=dWg, dWu=dWu, Gg=Gg, Gu=Gu, mu=mu, Qs=Qs).items()}
    return got, dict(X=X, R=R, w=w, Wg=Wg, Wu=Wu, dH=dH, dStream=dStream)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_whitened_block_end_to_end(dtype):
    got, i = whitened_step(dtype)
    # every step of the chain rounds to the type once; a result has at most eight such roundings behind it, added up without signs
    tol = 8 * HALF["bf16"] if dtype == "bf16" else 1e-5
    h = lo.f64(i["X"]) + lo.f64(i["R"])
    y = lo.rms_norm(h, i["w"], EPS)
    mu = y.mean(0)
    dY, dWg, dWu, _, _ = lo.gated_grad(y, i["Wg"], i["Wu"], "silu", i["dH"], mu=mu)
    dX, dw = lo.rms_norm_grad(h, i["w"], EPS, dY, i["dStream"])
    want = dict(H=h, Y=y, A=lo.gated(y, i["Wg"], i["Wu"], "silu"), dY=dY, dX=dX, dw=dw, dWg=dWg, dWu=dWu, mu=mu, Gg=dWg @ got["Qs"], Gu=dWu @ got["Qs"])
    for k, v in want.items():
        assert relF(got[k], v) < tol, k


def test_a_whitened_block_on_another_stream():
    side = torch.cuda.Stream()
    a, c = whitened_step("bf16")[0], whitened_step("bf16", side)[0]
    for k in a:
        assert np.array_equal(a[k], c[k]), k


def test_layers_captured_and_replayed():
    """Every call recorded into one graph; each replay on new contents of the same buffers gives what the eager calls give."""
    N, M, S, t, dt = 48, 200, 120, torch.bfloat16, b.FW_BF16
    rng = np.random.default_rng(8)
    d = b.conv_desc(N, M)
    e = lambda *s, k=t: torch.zeros(*s, dtype=k, device=DEV)  # noqa: E731
    X, R, dH = e(N, M), e(N, M), e(N, S)
    Wg, Wu, w = dev(rows(rng, S, M, "bf16", 0.1), t), dev(rows(rng, S, M, "bf16", 0.1), t), dev(np.ones(M, np.float32))
    Wq, sw = e(S, M, k=torch.int8), e(S, k=torch.float32)
    b.fw_int8_rows(Wg, dt, S, M, Wq, sw)
    ops = (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD, b.FW_OP_RMS_NORM_GRAD, b.FW_OP_INT8_PRODUCT)
    ws = [workspace(b.fw_workspace_bytes(op, M, S, d, dt)) for op in ops]

    def calls(o):
        b.fw_rms_norm(X, R, dt, N, M, w, EPS, o["H"], o["Y"], o["q"], o["qs"])
        b.fw_gated_forward(o["Y"], dt, N, M, S, Wg, Wu, None, None, b.FW_ACT_GELU, o["A"], o["Z"], ws[0])
        b.fw_gated_grad(o["Y"], dt, N, M, S, Wg, Wu, o["Z"], dH, w, o["dY"], o["dWg"], o["dWu"], o["dbg"], o["dbu"], ws[1])
        b.fw_rms_norm_grad(o["H"], dt, N, M, w, EPS, o["dY"], None, o["dX"], o["dw"], ws[2])
        b.fw_int8_product(o["q"], o["qs"], N, M, S, Wq, sw, None, o["P"], dt, ws[3])

    def outputs():
        f = torch.float32
        return dict(H=e(N, M), Y=e(N, M), q=e(N, M, k=torch.int8), qs=e(N, k=f), A=e(N, S), Z=e(2, N, S, k=f), dY=e(N, M), dWg=e(S, M), dWu=e(S, M), dbg=e(S),
                    dbu=e(S), dX=e(N, M), dw=e(M, k=f), P=e(N, S))

    eager, kept = outputs(), outputs()
    calls(kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(kept)
    for turn in range(3):
        for x, n in ((X, M), (R, M), (dH, S)):
            x.copy_(dev(rows(rng, N, n, "bf16"), t))
        calls(eager)
        torch.cuda.synchronize()
        for x in kept.values():
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(eager[k], kept[k]), (turn, k)
