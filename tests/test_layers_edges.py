"""Layers around the whitening, host side: memory that a call must not share, workspaces over all numbers of rows (no kernel runs)."""
import pytest

import layer_tiles as tiles
from paper_2010_01546_amd import binding as b

BASE, GAP = 1 << 20, 1 << 24          # aligned, never dereferenced: validation fails first

# arguments in order: (name, bytes for N rows, M features, S outputs of e bytes each) of those that point to memory, plain values otherwise;
# what a call writes; what an output may be in the place of
ROWS, WEIGHTS, RESULTS = (lambda N, M, S, e: N * M * e), (lambda N, M, S, e: S * M * e), (lambda N, M, S, e: N * S * e)
PER_N, PER_M, PER_S = (lambda N, M, S, e: 4 * N), (lambda N, M, S, e: 4 * M), (lambda N, M, S, e: 4 * S)
FACTORS, BIAS = (lambda N, M, S, e: 8 * N * S), (lambda N, M, S, e: e * S)
CALLS = {
    "fw_rms_norm": (dict(X=ROWS, R=ROWS, dt="dt", N="N", M="M", w=PER_M, eps=1e-5, H=ROWS, Y=ROWS, q=lambda N, M, S, e: N * M, qs=PER_N, stream=None),
                    ("H", "Y", "q", "qs"), {("H", "X"), ("H", "R")}, None),
    "fw_rms_norm_grad": (dict(H=ROWS, dt="dt", N="N", M="M", w=PER_M, eps=1e-5, dY=ROWS, dH=ROWS, dX=ROWS, dw=PER_M, ws="ws", n="n", stream=None),
                         ("dX", "dw", "ws"), {("dX", "dY"), ("dX", "dH")}, b.FW_OP_RMS_NORM_GRAD),
    "fw_gated_forward": (dict(X=ROWS, dt="dt", N="N", M="M", S="S", Wg=WEIGHTS, Wu=WEIGHTS, bg=PER_S, bu=PER_S, act=0, H=RESULTS, Z=FACTORS, ws="ws", n="n",
                              stream=None), ("H", "Z", "ws"), set(), b.FW_OP_GATED_FORWARD),
    "fw_gated_grad": (dict(X=ROWS, dt="dt", N="N", M="M", S="S", Wg=WEIGHTS, Wu=WEIGHTS, Z=FACTORS, dH=RESULTS, mu=PER_M, dX=ROWS, dWg=WEIGHTS, dWu=WEIGHTS,
                           dbg=BIAS, dbu=BIAS, ws="ws", n="n", stream=None), ("dX", "dWg", "dWu", "dbg", "dbu", "ws"), set(), b.FW_OP_GATED_GRAD),
    "fw_int8_rows": (dict(X=ROWS, dt="dt", N="N", M="M", q=lambda N, M, S, e: N * M, qs=PER_N, stream=None), ("q", "qs"), set(), None),
    "fw_int8_product": (dict(Xq=lambda N, M, S, e: N * M, sx=PER_N, N="N", M="M", S="S", Wq=lambda N, M, S, e: S * M, sw=PER_S, b=PER_S, Y=RESULTS, dt="dt",
                             ws="ws", n="n", stream=None), ("Y", "ws"), set(), b.FW_OP_INT8_PRODUCT),
}


@pytest.mark.parametrize("dt", [b.FW_F32, b.FW_BF16])
@pytest.mark.parametrize("name", CALLS)
def test_shared_memory_is_refused(name, dt):
    """Everything that a call writes, over the first and over the last bytes of everything else that it is given."""
    spec, written, may, op = CALLS[name]
    N, M, S, e = 96, 41, 72, 2 if dt == b.FW_BF16 else 4
    need = b.fw_workspace_bytes(op, M, S, b.conv_desc(N, M), dt) if op else 0
    values = dict(dt=dt, N=N, M=M, S=S, n=need)
    sizes = {k: v(N, M, S, e) for k, v in spec.items() if callable(v)}
    if op:
        assert need > 0
        sizes["ws"] = need
    at = {k: BASE + GAP * i for i, k in enumerate(sizes)}
    call = getattr(b.lib, name)
    seen = 0
    for out in written:
        for other in sizes:
            if other == out:
                continue
            # the output's first bytes over the other's last 16, its last bytes over the other's first, and both at one place
            for shift in (sizes[other] - 1) // 16 * 16, -((sizes[out] - 1) // 16 * 16), 0:
                if shift == 0 and (out, other) in may:
                    continue
                place = dict(at, **{out: at[other] + shift})
                args = [place[k] if k in place else values.get(v, v) if isinstance(v, str) else v for k, v in spec.items()]
                assert call(*args) == b.FW_ERR_INVALID_ARG, (out, other, shift)
                seen += 1
    assert seen > 5


@pytest.mark.parametrize("dt", [b.FW_F32, b.FW_BF16])
@pytest.mark.parametrize("op", [b.FW_OP_RMS_NORM_GRAD, b.FW_OP_GATED_FORWARD, b.FW_OP_GATED_GRAD, b.FW_OP_INT8_PRODUCT])
@pytest.mark.parametrize("M,S", [(64, 64), (33, 700), (576, 2304), (1153, 1001), (4608, 12288), (4609, 521)])
def test_a_workspace_is_enough_for_fewer_rows(M, S, op, dt):
    """No size is smaller than that of fewer rows; single rows around where forms change, odd steps between."""
    near = lambda n: range(max(1, n - 3), n + 4)  # noqa: E731
    N = sorted({*range(1, 140), *range(140, 9000, 37), *near(8192), *near((1 << 19) // S), *near(4096), *(64 * k + j for k in range(1, 40) for j in (0, 1))})
    sizes = [b.fw_workspace_bytes(op, M, S, b.conv_desc(n, M), dt) for n in N]
    assert all(x <= y for x, y in zip(sizes, sizes[1:]))


def test_sizes_reach_every_tile_and_cut():
    """What the tests on the GPU compare in full: every shape that a product is given, whole, cut into runs, and whole rounds with a cut rest
    behind them.  256 x 256 results (projections: 128 columns of both) are for two-byte and one-byte operands."""
    cuts = ("whole", "runs", "both")
    gates, plain = ("64x64", "64x128", "128x64", "128x128"), ("64x128", "64x256", "128x128", "128x256")
    for dt, sizes, largest in ((b.FW_BF16, tiles.BF16_SIZES, "256x256"), (b.FW_F32, tiles.F32_SIZES, None)):
        for product in ("forward", "dX", "dW"):
            shapes = list(gates if product == "forward" else plain) + ([largest.replace("x256", "x128") if product == "forward" else largest] if largest else [])
            if product == "dW":
                shapes.remove("64x256")                  # its rows are an even number of 64
            got = {tiles.way(tiles.choice(product, dt, *s)) for s in sizes}
            assert got - {None} == {(s, c) for s in shapes for c in cuts}, (dt, product)
    got = {tiles.way(tiles.choice("int8", b.FW_F32, *s)) for s in tiles.INT8_SIZES}
    assert got - {None} == {(s, c) for s in plain + ("256x256",) for c in cuts}


def test_few_rows_take_no_tiles():
    assert tiles.choice("forward", b.FW_F32, 32, 576, 200).few and tiles.choice("dW", b.FW_F32, 32, 576, 200).few and tiles.choice("int8", b.FW_F32, 16, 576, 200).few
    assert not tiles.choice("forward", b.FW_F32, 65, 576, 200).few and not tiles.choice("dX", b.FW_BF16, 1, 576, 200).few
