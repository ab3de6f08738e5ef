"""GPU parity of the layers around the whitening where a tie, an infinity or a size decides, against the float64 oracle.

Tolerances: U32 = 2^-24 and half(t) (2^-8 for bfloat16, 2^-24 for float32) are the most a rounding is off by, relative to its value."""
from fractions import Fraction

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
@pytest.mark.parametrize("N,M,S", [(60, 72, 130), (1000, 72, 520), (1030, 72, 520), (1030, 75, 523)])
def test_infinite_gradients_of_centred_rows(N, M, S, dtype):
    """With mu, an infinite dg or du makes its row of dWg or dWu infinite with the sign that X - mu has, and NaN where X - mu is zero; in
    bfloat16 on both sides of the 524288 entries from which on dg and du are one number."""
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
