"""GPU parity of the layers around the whitening where a tie, an infinity or a size decides, against the float64 oracle.

Tolerances: U32 = 2^-24 and half(t) (2^-8 for bfloat16, 2^-24 for float32) are the most a rounding is off by, relative to its value."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import layer_tiles as tiles
import workloads as wl
from gpu_common import DEV, b, dev, relF, workspace
from oracle import layer_oracle as lo
from test_gpu_layers import Out

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
FDT = {"f32": b.FW_F32, "bf16": b.FW_BF16}
EPS = 1e-5


def nearest_even(v, top):
    """127 v / top to the nearest integer, ties to even, in whole numbers."""
    return round(Fraction(127) * v / top)


def held(x, dtype):
    x = np.array([x], dtype=np.float32)
    return float((wl.round_to_bf16(x) if dtype == "bf16" else x)[0])


def step(x, dtype, up):
    """The next number of the type."""
    if dtype == "f32":
        return np.nextafter(np.float32(x), np.float32(np.inf if up else -np.inf))
    bits = np.float32(x).view(np.uint32) >> 16
    return np.uint32(int(bits) + (1 if up == (x > 0) else -1) << 16).view(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_of_8_bit_rows(dtype):
    """Entries halfway between two steps go to the even one, their neighbours to the nearer one: for every bfloat16 significand of the row's
    largest entry, and (float32) for 24-bit ones, of which the multiples of 127 have ties at every step."""
    tops = [float(t) for t in range(128, 256)]
    if dtype == "f32":
        rng = np.random.default_rng(17)
        tops += [float(2 * t) for t in rng.integers(1 << 22, 1 << 23, 64)] + [float(254 * t) for t in rng.integers(1 << 13, 1 << 16, 64)]
    X = np.zeros((len(tops), 268), dtype=np.float32)
    for row, top in zip(X, tops):
        halves = [(2 * j + 1) * top / 254 for j in range(127)]
        halves = [x for x in halves if held(x, dtype) == x and Fraction(x) * 254 % Fraction(top) == 0]
        assert top / 2 in halves
        entries = [top] + [s * x for x in halves for s in (1, -1)]
        entries += [step(s * x, dtype, up) for x in halves[-1:] + [top / 2] for s in (1, -1) for up in (False, True)]
        row[:len(entries)] = entries
    N, M = X.shape
    want = np.array([[nearest_even(Fraction(float(x)), Fraction(t)) for x in row] for row, t in zip(X, tops)])
    q, qs, q2, qs2 = (torch.zeros(s, dtype=k, device=DEV) for s, k in (((N, M), torch.int8), (N, torch.float32)) * 2)
    b.fw_int8_rows(dev(X, TDT[dtype]), FDT[dtype], N, M, q, qs)
    b.fw_rms_norm(dev(X, TDT[dtype]), None, FDT[dtype], N, M, None, EPS, None, None, q2, qs2)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), want)
    assert np.array_equal(q2.cpu().numpy(), want)


def test_ties_of_products_with_the_weights():
    """h w of 48 bits: halves of the largest one are ties, products a 2^-46th below are not."""
    rng = np.random.default_rng(18)
    N, M = 200, 9
    a = rng.integers(1 << 23, (1 << 24) - 1, N).astype(np.float32)
    c = np.float32(rng.integers(1 << 23, (1 << 24) - 1)) * np.float32(2.0 ** -24)
    w = np.full(M, c, dtype=np.float32)
    w[1:3], w[3], w[4:] = c / 2, np.nextafter(c / 2, np.float32(0)), c / 4
    X = np.zeros((N, M), dtype=np.float32)
    X[:, 0], X[:, 1], X[:, 2], X[:, 3] = a, a, -a, a + 1
    X[:, 3] = np.where((a + 1) * w[3].astype(np.float64) <= a * lo.f64(c), X[:, 3], a)
    X[:, 4:] = (rng.integers(1, 1 << 24, (N, M - 4)) // 2).astype(np.float32)
    v = [[Fraction(float(x)) * Fraction(float(y)) for x, y in zip(row, w)] for row in X]
    top = [max(abs(x) for x in row) for row in v]
    want = np.array([[nearest_even(x, t) for x in row] for row, t in zip(v, top)])
    assert (want[:, 1] == 64).all() and (want[:, 2] == -64).all() and (want[:, 3] == 63).any()
    q, qs = torch.zeros(N, M, dtype=torch.int8, device=DEV), torch.zeros(N, device=DEV)
    b.fw_rms_norm(dev(X), None, b.FW_F32, N, M, dev(w), EPS, None, None, q, qs)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", [(60, 72, 130), (1000, 72, 520), (1030, 72, 520), (1030, 75, 523), (600, 1300, 1000), (517, 545, 6559), (1300, 2000, 3000)])
def test_infinite_gradients_of_centred_rows(N, M, S, dtype):
    """With mu, an infinite dg or du makes its row of dWg or dWu infinite with the sign that X - mu has, and NaN where X - mu is zero; in
    bfloat16 on both sides of the 524288 entries from which on dg and du are one number, in tiles cut into runs, whole ones, and both."""
    t, dt = TDT[dtype], FDT[dtype]
    rng = np.random.default_rng(N + M)
    low = wl.round_to_bf16 if dtype == "bf16" else (lambda x: x)
    X, Wg, Wu, dH = (low(rng.standard_normal(s).astype(np.float32)) for s in ((N, M), (S, M), (S, M), (N, S)))
    mu = X.mean(0).astype(np.float32)
    mu[:5] = 0.0
    X[3, 7] = mu[7] = 0.25                                       # X - mu = 0 in an infinite row: NaN
    Z = (0.3 + np.abs(rng.standard_normal((2, N, S)))).astype(np.float32)
    dH[3, 9], dH[N - 2, S - 1] = np.inf, -np.inf
    dX, dWg, dWu = (torch.empty(s, dtype=t, device=DEV) for s in ((N, M), (S, M), (S, M)))
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    ws.fill_(255)
    b.fw_gated_grad(dev(X, t), dt, N, M, S, dev(Wg, t), dev(Wu, t), dev(Z), dev(dH, t), dev(mu), dX, dWg, dWu, None, None, ws)
    torch.cuda.synchronize()
    D = [lo.f64(dH) * Z[k] for k in range(2)]
    with np.errstate(all="ignore"):
        want = lo.gated_grad_from(D[0], D[1], X, Wg, Wu, mu)
    for got, w, what in zip((dX, dWg, dWu), want, ("dX", "dWg", "dWu")):
        got = got.float().cpu().numpy().astype(np.float64)
        fine = np.isfinite(w)
        assert np.array_equal(np.isnan(got), np.isnan(w)), what
        assert np.array_equal(got[np.isinf(w)], w[np.isinf(w)]), what
        # two roundings to the type, of dg or du and of the result
        assert fine.any() and relF(got[fine], w[fine]) < (2 * HALF["bf16"] if dtype == "bf16" else 1e-5), what


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_workspace_for_all_numbers_of_rows(dtype):
    """A workspace of the largest batch, as a program keeps it: smaller ones run in it and give what they give in their own."""
    most, M, S, t, dt = 1500, 580, 900, TDT[dtype], FDT[dtype]
    rng = np.random.default_rng(3)
    X, Wg, Wu, dH = (dev(rng.standard_normal(s).astype(np.float32) / 8, t) for s in ((most, M), (S, M), (S, M), (most, S)))
    Xq, Wq = (dev(rng.integers(-127, 128, s), torch.int8) for s in ((most, M), (S, M)))
    scale = torch.ones(most, device=DEV)
    ops = (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD, b.FW_OP_RMS_NORM_GRAD, b.FW_OP_INT8_PRODUCT)
    space = lambda N: [torch.full((b.fw_workspace_bytes(op, M, S, b.conv_desc(N, M), dt),), 255, dtype=torch.uint8, device=DEV) for op in ops]  # noqa: E731

    def run(N, ws):
        H, Z, dX, dY = (torch.empty(s, dtype=k, device=DEV) for s, k in (((N, S), t), ((2, N, S), torch.float32), ((N, M), t), ((N, M), t)))
        dWg, dWu, dw, Y = (torch.empty(s, dtype=k, device=DEV) for s, k in (((S, M), t), ((S, M), t), ((M,), torch.float32), ((N, S), t)))
        b.fw_gated_forward(X, dt, N, M, S, Wg, Wu, None, None, b.FW_ACT_SILU, H, Z, ws[0])
        b.fw_gated_grad(X, dt, N, M, S, Wg, Wu, Z, dH, None, dX, dWg, dWu, None, None, ws[1])
        b.fw_rms_norm_grad(X, dt, N, M, None, EPS, dX, None, dY, dw, ws[2])
        b.fw_int8_product(Xq, scale, N, M, S, Wq, scale, None, Y, dt, ws[3])
        torch.cuda.synchronize()
        return H, Z, dX, dY, dWg, dWu, dw, Y

    kept = space(most)
    for N in (most, 1, 16, 17, 40, 64, 65, 200, (1 << 19) // S, (1 << 19) // S + 1, 700, 1024, 1499):
        for a, c in zip(run(N, kept), run(N, space(N))):
            assert torch.equal(a, c), N


@pytest.mark.parametrize("N,M,S", [(1030, 75, 523), (600, 1300, 1000)])
def test_nan_and_infinite_gradients_of_centred_rows(N, M, S):
    """bfloat16, dg and du as one number: columns with a NaN, with infinities of one sign and of both, and a mean that is not finite."""
    t, dt = torch.bfloat16, b.FW_BF16
    rng = np.random.default_rng(N)
    X, Wg, Wu, dH = (wl.round_to_bf16(rng.standard_normal(s).astype(np.float32)) for s in ((N, M), (S, M), (S, M), (N, S)))
    mu = (X.mean(0) + 0.05).astype(np.float32)
    Z = (0.3 + np.abs(rng.standard_normal((2, N, S)))).astype(np.float32)
    dH[N - 1, 0], dH[0, 1], dH[5, 2:20] = np.nan, np.nan, np.inf
    dH[7, 3], dH[N // 2, 40], dH[2, 41], dH[3, 41] = -np.inf, np.inf, np.inf, np.nan
    Z[1, 4, 60] = np.nan                                          # in du alone
    mu[11] = np.inf
    dWg, dWu = (torch.empty(S, M, dtype=t, device=DEV) for _ in range(2))
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    b.fw_gated_grad(dev(X, t), dt, N, M, S, dev(Wg, t), dev(Wu, t), dev(Z), dev(dH, t), dev(mu), None, dWg, dWu, None, None, ws)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        want = lo.gated_grad_from(lo.f64(dH) * Z[0], lo.f64(dH) * Z[1], X, Wg, Wu, mu)
    for got, w, what in zip((dWg, dWu), want[1:3], ("dWg", "dWu")):
        got = got.float().cpu().numpy().astype(np.float64)
        fine = np.isfinite(w)
        assert np.array_equal(np.isnan(got), np.isnan(w)) and np.array_equal(got[np.isinf(w)], w[np.isinf(w)]), what
        assert fine.any() and relF(got[fine], w[fine]) < 2 * HALF["bf16"], what


def test_time_of_nan_gradients_of_centred_rows():
    """A step full of NaN, as a diverged loss leaves it, takes about as long as any other: nothing is computed again for it."""
    N, M, S, t, dt = 1000, 4608, 4000, torch.bfloat16, b.FW_BF16
    X, W = torch.ones(N, M, device=DEV, dtype=t), torch.ones(S, M, device=DEV, dtype=t)
    Z, dH, mu = torch.ones(2, N, S, device=DEV), torch.full((N, S), float("nan"), device=DEV, dtype=t), torch.ones(M, device=DEV)
    dWg, dWu = torch.empty_like(W), torch.empty_like(W)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_GATED_GRAD, M, S, b.conv_desc(N, M), dt))
    begin, end = torch.cuda.Event(True), torch.cuda.Event(True)
    for turn in range(2):
        begin.record()
        b.fw_gated_grad(X, dt, N, M, S, W, W, Z, dH, mu, None, dWg, dWu, None, None, ws)
        end.record()
        torch.cuda.synchronize()
    assert bool(torch.isnan(dWg).all()) and bool(torch.isnan(dWu).all())
    assert begin.elapsed_time(end) < 3                             # ms; 0.13 of finite ones, 6 where everything is computed again


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M,S", [(5, 64, 70), (200, 144, 300)])
def test_scales_far_from_one(N, M, S, dtype):
    """A sum times its token's scale may lie outside float32 where the result does not."""
    rng = np.random.default_rng(N)
    Xq, Wq = rng.integers(-127, 128, (N, M)).astype(np.int8), rng.integers(-127, 128, (S, M)).astype(np.int8)
    sx = (np.exp(rng.standard_normal(N)) * np.where(np.arange(N) % 2, 1e36, 1e-36)).astype(np.float32)
    sw = (np.exp(rng.standard_normal(S)) * np.where(np.arange(S) % 3, 1e-7, 1e-30)).astype(np.float32)
    Xq[0] = 0                                                    # 0 times anything finite
    Y = torch.empty(N, S, dtype=TDT[dtype], device=DEV)
    ws = workspace(b.fw_workspace_bytes(b.FW_OP_INT8_PRODUCT, M, S, b.conv_desc(N, M), FDT[dtype]))
    b.fw_int8_product(dev(Xq, torch.int8), dev(sx), N, M, S, dev(Wq, torch.int8), dev(sw), None, Y, FDT[dtype], ws)
    torch.cuda.synchronize()
    want = lo.int8_product(Xq, sx, Wq, sw)
    got = Y.float().cpu().numpy().astype(np.float64)
    assert np.abs(want).max() < 3e38 and np.isfinite(got).all()
    # the sum's and both products' roundings and the type's; below 2^-126 a float32 number is off by up to 2^-150
    assert (np.abs(got - want) <= 4 * U32 * np.abs(want) + HALF[dtype] * np.abs(want) + 2.0 ** -133).all()


# ------------------------------------------------------------------------------- every tile and cut, all results, in float64 on the GPU

def within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i].item()!r} for {want[i].item()!r}, allowed {tol[i].item():.3g}")


def close(got, want, roundings, what):
    """float32, as a whole: the roundings of a sum of K terms of either sign are each at most U32 of a partial sum, which is no larger than
    the whole one in the mean of squares, and of either sign, so that sqrt(K) of them remain.  (One of six products of the three
    planes left out is 2^-18.)"""
    rel = (torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want)).item()
    assert rel < roundings * U32, (what, rel, roundings * U32)


def untouched(*outs):
    for x in outs:
        tail = x.buf[x.t.numel():].float()
        assert bool((tail == 77).all() if x.fill == 77 else torch.isnan(tail).all()), "written behind the end"


@pytest.mark.parametrize("dtype,N,M,S", [("bf16", *s) for s in tiles.BF16_SIZES] + [("f32", *s) for s in tiles.F32_SIZES])
def test_gated_block_of_every_tile(dtype, N, M, S):
    t, dt, half = TDT[dtype], FDT[dtype], HALF[dtype]
    gen = torch.Generator(device=DEV).manual_seed(N + M + S)
    new = lambda *s, scale=1.0: scale * torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    X = (new(N, M) * torch.exp(0.5 * new(M))).to(t)
    Wg, Wu, dH = (new(*s, scale=c).to(t) for s, c in (((S, M), M ** -0.5), ((S, M), M ** -0.5), ((N, S), 0.1)))
    bg, bu = new(S, scale=0.3), new(S, scale=0.3)
    mu = X.float().mean(0) + 0.1 if (N + M) % 4 else None
    H, Z = Out(N, S, dtype=t), Out(2, N, S, dtype=torch.float32)
    dX, dWg, dWu, dbg, dbu = (Out(*s, dtype=t) for s in ((N, M), (S, M), (S, M), (S,), (S,)))
    d = b.conv_desc(N, M)
    ws = [torch.full((max(b.fw_workspace_bytes(op, M, S, d, dt), 16),), 255, dtype=torch.uint8, device=DEV) for op in (b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD)]
    b.fw_gated_forward(X, dt, N, M, S, Wg, Wu, bg, bu, b.FW_ACT_SILU, H.t, Z.t, ws[0])
    b.fw_gated_grad(X, dt, N, M, S, Wg, Wu, Z.t, dH, mu, dX.t, dWg.t, dWu.t, dbg.t, dbu.t, ws[1])
    torch.cuda.synchronize()
    untouched(H, Z, dX, dWg, dWu, dbg, dbu)
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    g, u = x @ wg.T + bg, x @ wu.T + bu
    # a sum of K terms in float32, in any order, is off by (K + a few) U32 of the terms' magnitudes; slopes of silu and of its slope are
    # below 1.2; the activation is off by a few units of float32 of max(|g|, 1)
    eg, eu = ((M + 8) * U32 * (x.abs() @ w.abs().T + c.abs()) for w, c in ((wg, bg), (wu, bu)))
    p = torch.sigmoid(g)
    a, da = g * p, p + g * p * (1 - p)
    within(H.t, a * u, 1.2 * eg * (u.abs() + eu) + a.abs() * eu + 16 * U32 * (g * u).abs() + (a * u).abs() * half + 1e-38, "H")
    within(Z.t[0], u * da, 1.2 * eg * u.abs() + 1.2 * eu + 16 * U32 * (1 + g.abs()) * u.abs() + 1e-38, "Z[0]")
    within(Z.t[1], a, 1.2 * eg + 16 * U32 * g.abs() + 1e-38, "Z[1]")
    if dtype == "f32":       # slope 1.2 of an activation half as large in the mean of squares, and the other factor's own error
        close(H.t, a * u, 4 * M ** 0.5 + 32, "H")
        close(Z.t[1], a, 3 * M ** 0.5 + 32, "Z[1]")
    del g, u, p, a, da, eg, eu
    # the gradients of what was kept: dg and du in float32, in bfloat16 rounded to one number where there are many, to two otherwise
    one = dtype == "bf16" and N * S > 1 << 19
    more = U32 if dtype == "f32" else 0.0 if one else U32 + 2.0 ** -16
    D = [dH.float() * Z.t[k] for k in range(2)]
    for got, v, what in ((dbg, D[0], "dbg"), (dbu, D[1], "dbu")):
        within(got.t, v.double().sum(0), (N + 5) * U32 * v.double().abs().sum(0) + half * v.double().sum(0).abs(), what)
    D = [v.to(t).double() if one else v.double() for v in D]
    want = D[0] @ wg + D[1] @ wu
    within(dX.t, want, ((2 * S + 8) * U32 + more) * (D[0].abs() @ wg.abs() + D[1].abs() @ wu.abs()) + half * want.abs(), "dX")
    if dtype == "f32":
        close(dX.t, want, (2 * S) ** 0.5 + 8, "dX")
    xc, xm = (x, x.abs()) if mu is None else (x - mu, x.abs() + mu.abs())
    for got, v, what in ((dWg, D[0], "dWg"), (dWu, D[1], "dWu")):
        want = v.T.contiguous() @ xc
        within(got.t, want, ((2 * N + 8) * U32 + more) * (v.abs().T.contiguous() @ xm.double()) + half * want.abs(), what)
        if dtype == "f32":
            close(got.t, want, N ** 0.5 + 8, what)


@pytest.mark.parametrize("N,M,S", tiles.INT8_SIZES)
def test_int8_product_of_every_tile(N, M, S):
    gen = torch.Generator(device=DEV).manual_seed(N + M + S)
    Xq, Wq = (torch.randint(-127, 128, s, generator=gen, device=DEV, dtype=torch.int8) for s in ((N, M), (S, M)))
    sx, sw = (torch.exp(torch.randn(n, generator=gen, device=DEV)) for n in (N, S))
    bias = torch.randn(S, generator=gen, device=DEV)
    Y = Out(N, S, dtype=torch.float32)
    ws = torch.full((max(b.fw_workspace_bytes(b.FW_OP_INT8_PRODUCT, M, S, b.conv_desc(N, M), b.FW_F32), 16),), 255, dtype=torch.uint8, device=DEV)
    b.fw_int8_product(Xq, sx, N, M, S, Wq, sw, bias, Y.t, b.FW_F32, ws)
    torch.cuda.synchronize()
    untouched(Y)
    plain = (Xq.double() @ Wq.double().T) * sx.double()[:, None] * sw.double()
    within(Y.t, plain + bias, 4 * U32 * (plain.abs() + bias.abs()), "Y")
