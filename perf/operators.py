"""Operators around a whitened layer of a language model, as cases that can be timed and compared: the norm that makes the layer's
input rows, the gated feed-forward block whose backward pass makes the weight gradients, and the 8-bit product that answers with
the trained weights.

  norm    H = X + R held in the inputs' type, Y = rows of H over their root mean square, times w
  norm8   the same with Y in 8 bits and a scale per row; compared as the values it stands for
  normgrad  gradient of the norm with respect to H and w, the residual path's gradient added
  gated   H = act(X Wg^T + bg) * (X Wu^T + bu)
  train   the same and its backward pass: H, dX, dWg, dWu (centred on mu where the layer is), and the biases' gradients
  int8    Y = Xq Wq^T times the rows' and the channels' scales (+ b); with `quantise` the rows come in the activations' type

With `own` false the passes are computed by elementary torch operations in 32 bits, otherwise through the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


def _norm(name, kind, N, M, dtype, residual=True):
    c = {"kind": kind, "N": N, "M": M, "dtype": dtype, "residual": residual}
    return dict(c, name=name) if name else c


def _gated(name, kind, N, M, S, dtype, act="silu", bias=False, centred=False):
    c = {"kind": kind, "N": N, "M": M, "S": S, "dtype": dtype, "act": act, "bias": bias, "centred": centred}
    return dict(c, name=name) if name else c


def _int8(name, N, M, S, dtype, quantise=False, bias=False):
    c = {"kind": "int8", "N": N, "M": M, "S": S, "dtype": dtype, "quantise": quantise, "bias": bias}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of an answer: the smallest call, all latency
        _norm("norm-1x4608", "norm", 1, 4608, "bf16"),
        # a training batch of 8192 tokens
        _norm("norm-8192x4608", "norm", 8192, 4608, "bf16"),
        # a prompt ahead of an 8-bit layer, odd width and length
        _norm("norm8-1531x2305", "norm8", 1531, 2305, "bf16"),
        # backward pass of the training batch in float32, as a small model trains
        _norm("normgrad-4096x1152", "normgrad", 4096, 1152, "f32"),
        # backward pass of the training batch, bfloat16
        _norm("normgrad-8192x4608", "normgrad", 8192, 4608, "bf16"),
        # one token through the gated block: reads both weight matrices once
        _gated("gated-1x4608x12288", "gated", 1, 4608, 12288, "bf16"),
        # a prompt of odd length through a block of odd sizes, with biases
        _gated("gated-501x2304x6145", "gated", 501, 2304, 6145, "bf16", "gelu", bias=True),
        # training step of a small float32 layer, whitened: centred gradients and biases
        _gated("train-1024x576x2304-f32", "train", 1024, 576, 2304, "f32", bias=True, centred=True),
        # training step of a ragged batch, every size odd
        _gated("train-777x1153x1001", "train", 777, 1153, 1001, "bf16", "gelu_tanh", bias=True, centred=True),
        # training step of 8192 tokens: the largest call
        _gated("train-8192x4608x12288", "train", 8192, 4608, 12288, "bf16"),
        # a batch of sixteen answers through the projection back, rows to 8 bits in the call
        _int8("int8-16x12288x4608", 16, 12288, 4608, "bf16", quantise=True),
        # a long prompt in 8 bits
        _int8("int8-8192x4608x12288", 8192, 4608, 12288, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths as layers have them, multiples of 64 or 8, and odd ones."""
    n = _log_int(rng, lo, hi)
    m = rng.choice([64, 64, 8, 1])
    return max(m, n // m * m)


def draw(rng):
    kind = rng.choice(["norm", "norm8", "normgrad", "gated", "gated", "train", "train", "int8", "int8"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    N = _log_int(rng, 1, 8192)
    if kind in ("norm", "norm8", "normgrad"):
        return _norm(None, kind, N, _width(rng, 48, 4608), dtype, rng.random() < 0.75)
    if kind == "int8":
        return _int8(None, N, _width(rng, 48, 4608), _width(rng, 48, 12288), dtype, rng.random() < 0.5, rng.random() < 0.3)
    while True:
        M, S = _width(rng, 48, 4608), _width(rng, 48, 12288)
        # float32 products run at a small part of the bfloat16 rate: smaller layers
        if dtype == "bf16" or N * M * S <= 1 << 36:
            break
        N = _log_int(rng, 1, 8192)
    bias = rng.random() < 0.4
    return _gated(None, kind, N, M, S, dtype, rng.choice(["silu", "silu"] + ACTS[1:]), bias, kind == "train" and rng.random() < 0.4)


def _tdt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, n, m, dtype, scale=1.0):
    """Rows with correlated size: channels of unequal power (a few large ones) and tokens of unequal norm."""
    ch = torch.exp(0.5 * torch.randn(m, generator=g, device=DEV))
    tok = torch.exp(0.2 * torch.randn(n, 1, generator=g, device=DEV))
    return (torch.randn(n, m, generator=g, device=DEV).mul_(ch).mul_(tok).mul_(scale)).to(dtype)


def _quantised(x):
    """Rows in 8 bits with a scale each, as a program stores its weights."""
    x = x.float()
    s = x.abs().amax(1) / 127
    return torch.round(x / s.clamp_min(1e-30)[:, None]).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, N, M, t = case["kind"], case["N"], case["M"], _tdt(case)
    st = {"case": case}
    new = lambda *shape, dt=t: torch.empty(*shape, dtype=dt, device=DEV)  # noqa: E731
    if kind in ("norm", "norm8", "normgrad"):
        st["w"] = 1 + 0.1 * torch.randn(M, generator=g, device=DEV)
        st["X"] = _rows(g, N, M, t)
        if case["residual"]:
            st["R"] = _rows(g, N, M, t, 1e-2 if kind == "normgrad" else 2.0)
        if kind == "normgrad":
            st["dY"] = _rows(g, N, M, t, 1e-2)
    elif kind == "int8":
        S = case["S"]
        x = _rows(g, N, M, t)
        if case["quantise"]:
            st["X"] = x
        else:
            st["Xq"], st["sx"] = _quantised(x)
        st["Wq"], st["sw"] = _quantised(torch.randn(S, M, generator=g, device=DEV) * M ** -0.5)
        st["b"] = 0.1 * torch.randn(S, generator=g, device=DEV) if case["bias"] else None
    else:
        S = case["S"]
        st["X"] = _rows(g, N, M, t, 0.7)
        if case["centred"]:      # rows with a mean, which the layer's whitening takes out of the gradient
            st["X"] = (st["X"].float() + 0.3 * torch.randn(M, generator=g, device=DEV)).to(t)
            st["mu"] = st["X"].float().mean(0)
        st["Wg"] = (torch.randn(S, M, generator=g, device=DEV) * M ** -0.5).to(t)
        st["Wu"] = (torch.randn(S, M, generator=g, device=DEV) * M ** -0.5).to(t)
        if case["bias"]:
            st["bg"], st["bu"] = (0.1 * torch.randn(S, generator=g, device=DEV) for _ in range(2))
        if kind == "train":
            st["dH"] = _rows(g, N, S, t, 1e-2)
    if own:
        _keep(st, case, new)
    return st


def _keep(st, case, new):
    """Outputs and workspaces that a program keeps from call to call."""
    from paper_2010_01546_amd import binding as fw
    kind, N, M = case["kind"], case["N"], case["M"]
    dt = st["dt"] = fw.FW_BF16 if case["dtype"] == "bf16" else fw.FW_F32
    d = fw.conv_desc(N, M)
    space = lambda *a: new(max(fw.fw_workspace_bytes(*a), 16), dt=torch.uint8)  # noqa: E731
    if kind == "norm":
        st["Y"], st["H"] = new(N, M), new(N, M) if case["residual"] else None
    elif kind == "norm8":
        st["q"], st["qs"] = new(N, M, dt=torch.int8), new(N, dt=torch.float32)
        st["H"] = new(N, M) if case["residual"] else None
    elif kind == "normgrad":
        st["dX"], st["dw"] = new(N, M), new(M, dt=torch.float32)
        st["ws"] = space(fw.FW_OP_RMS_NORM_GRAD, M, 0, d, dt)
    elif kind == "int8":
        S = case["S"]
        st["Y"] = new(N, S)
        if case["quantise"]:
            st["Xq"], st["sx"] = new(N, M, dt=torch.int8), new(N, dt=torch.float32)
        st["ws"] = space(fw.FW_OP_INT8_PRODUCT, M, S, d, dt)
    else:
        S = case["S"]
        st["act"] = [fw.FW_ACT_SILU, fw.FW_ACT_GELU, fw.FW_ACT_GELU_TANH, fw.FW_ACT_RELU][ACTS.index(case["act"])]
        st["H"] = new(N, S)
        st["ws"] = space(fw.FW_OP_GATED_FORWARD, M, S, d, dt)
        if kind == "train":
            st["Z"] = new(2, N, S, dt=torch.float32)
            st["dX"], st["dWg"], st["dWu"] = new(N, M), new(S, M), new(S, M)
            if case["bias"]:
                st["dbg"], st["dbu"] = new(S), new(S)
            st["ws_grad"] = space(fw.FW_OP_GATED_GRAD, M, S, d, dt)


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2010_01546_amd import binding as fw
    case, dt = st["case"], st["dt"]
    kind, N, M = case["kind"], case["N"], case["M"]
    if kind == "norm":
        fw.fw_rms_norm(st["X"], st.get("R"), dt, N, M, st["w"], EPS, st["H"], st["Y"], None, None)
        return [st["Y"], st["H"]] if case["residual"] else [st["Y"]]
    if kind == "norm8":
        fw.fw_rms_norm(st["X"], st.get("R"), dt, N, M, st["w"], EPS, st["H"], None, st["q"], st["qs"])
        y = torch.mul(st["q"], st["qs"][:, None])
        return [y, st["H"]] if case["residual"] else [y]
    if kind == "normgrad":
        fw.fw_rms_norm_grad(st["X"], dt, N, M, st["w"], EPS, st["dY"], st.get("R"), st["dX"], st["dw"], st["ws"])
        return [st["dX"], st["dw"]]
    S = case["S"]
    if kind == "int8":
        if case["quantise"]:
            fw.fw_int8_rows(st["X"], dt, N, M, st["Xq"], st["sx"])
        fw.fw_int8_product(st["Xq"], st["sx"], N, M, S, st["Wq"], st["sw"], st["b"], st["Y"], dt, st["ws"])
        return [st["Y"]]
    fw.fw_gated_forward(st["X"], dt, N, M, S, st["Wg"], st["Wu"], st.get("bg"), st.get("bu"), st["act"], st["H"], st.get("Z"), st["ws"])
    if kind == "gated":
        return [st["H"]]
    fw.fw_gated_grad(st["X"], dt, N, M, S, st["Wg"], st["Wu"], st["Z"], st["dH"], st.get("mu"), st["dX"], st["dWg"],
                     st["dWu"], st.get("dbg"), st.get("dbu"), st["ws_grad"])
    return [st[k] for k in ("H", "dX", "dWg", "dWu") + (("dbg", "dbu") if case["bias"] else ())]


def _act(kind, g):
    """Value and derivative."""
    if kind == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        p = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    if kind == "gelu_tanh":
        k = (2 / math.pi) ** 0.5
        th = torch.tanh(k * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * k * (1 + 3 * 0.044715 * g * g)
    return torch.where(g > 0, g, torch.zeros_like(g)), (g > 0).to(g.dtype)


def _to8(x):
    """Rows in steps of a 127th of their largest entry."""
    s = x.abs().amax(1, keepdim=True) / 127
    return torch.where(s > 0, torch.round(x / s), torch.zeros_like(x)), s


def _run_plain(st):
    case, t = st["case"], _tdt(st["case"])
    kind = case["kind"]
    if kind in ("norm", "norm8"):
        h = (st["X"].float() + st["R"].float()).to(t) if case["residual"] else st["X"]
        y = h.double() if kind == "norm8" else h.float()       # in 64 bits: a value next to a rounding's border
        y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * st["w"]
        if kind == "norm8":
            y, s = _to8(y)
            y = (y * s).float()
        else:
            y = y.to(t)
        return [y, h] if case["residual"] else [y]
    if kind == "normgrad":
        h, dy = st["X"].float(), st["dY"].float()
        rho = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        wdy = dy * st["w"]
        dx = rho * wdy - h * (rho ** 3 * (wdy * h).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + st["R"].float()
        return [dx.to(t), (dy * h * rho).sum(0)]
    if kind == "int8":
        xq, sx = st["Xq"].float() if not case["quantise"] else None, st.get("sx")
        if case["quantise"]:
            xq, sx = _to8(st["X"].double())
            xq, sx = xq.float(), sx[:, 0].float()
        y = (xq @ st["Wq"].float().T) * sx[:, None] * st["sw"]
        return [(y if st["b"] is None else y + st["b"]).to(t)]
    x, wg, wu = st["X"].float(), st["Wg"].float(), st["Wu"].float()
    g, u = x @ wg.T, x @ wu.T
    if case["bias"]:
        g, u = g + st["bg"], u + st["bu"]
    a, da = _act(case["act"], g)
    h = (a * u).to(t)
    if kind == "gated":
        return [h]
    dh = st["dH"].float()
    dg, du = dh * u * da, dh * a
    dx = dg @ wg + du @ wu
    if case["centred"]:
        x = x - st["mu"]
    out = [h, dx.to(t), (dg.T @ x).to(t), (du.T @ x).to(t)]
    return out + [dg.sum(0).to(t), du.sum(0).to(t)] if case["bias"] else out


def exact(case, seed):
    """The definitions in 64 bits, a block of rows at a time where that is enough."""
    st = prepare(case, seed)
    d = lambda k: st[k].double()  # noqa: E731
    kind, t = case["kind"], _tdt(case)
    if kind in ("norm", "norm8"):
        h = (d("X") + d("R")).to(t) if case["residual"] else st["X"]
        y = h.double() / (h.double().pow(2).sum(1, keepdim=True) / case["M"] + EPS).sqrt() * d("w")
        if kind == "norm8":
            top = y.abs().max(1, keepdim=True).values
            y = (y * 127 / top.clamp_min(1e-300)).round() * top / 127
        return [y, h.double()] if case["residual"] else [y]
    if kind == "normgrad":
        h, dy = d("X"), d("dY")
        r = (h.pow(2).sum(1, keepdim=True) / case["M"] + EPS).sqrt()
        n = h / r
        v = dy * d("w")
        dx = (v - n * (v * n).sum(1, keepdim=True) / case["M"]) / r
        return [dx + d("R") if case["residual"] else dx, (dy * n).sum(0)]
    if kind == "int8":
        if case["quantise"]:
            top = d("X").abs().max(1, keepdim=True).values
            x = (d("X") * 127 / top.clamp_min(1e-300)).round() * (top / 127)
        else:
            x = d("Xq") * d("sx")[:, None]
        w = d("Wq") * d("sw")[:, None]
        y = torch.cat([x[i:i + 2048] @ w.T for i in range(0, case["N"], 2048)])
        return [y + d("b") if case["bias"] else y]
    N, M, S = case["N"], case["M"], case["S"]
    f64 = dict(dtype=torch.float64, device=DEV)
    wg, wu = d("Wg"), d("Wu")
    mu = d("mu") if case["centred"] else torch.zeros(M, **f64)
    hs, dxs = [], []
    Gg, Gu, sg, su = torch.zeros(S, M, **f64), torch.zeros(S, M, **f64), torch.zeros(S, **f64), torch.zeros(S, **f64)
    for i in range(0, N, 2048):
        x = st["X"][i:i + 2048].double()
        g, u = x @ wg.T, x @ wu.T
        if case["bias"]:
            g += d("bg")
            u += d("bu")
        if case["act"] == "silu":
            c = torch.sigmoid(g)
            slope = c + g * c * (1 - c)
        elif case["act"] == "gelu":
            c = 0.5 * torch.erfc(-g / math.sqrt(2))
            slope = c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        elif case["act"] == "gelu_tanh":
            k = math.sqrt(2 / math.pi)
            z = k * (g + 0.044715 * g ** 3)
            c = torch.sigmoid(2 * z)                       # (1 + tanh z) / 2
            slope = c + 2 * g * c * (1 - c) * k * (1 + 0.134145 * g * g)
        else:
            c = (g > 0).double()
            slope = c
        hs.append(g * c * u)
        if kind == "gated":
            continue
        dh = st["dH"][i:i + 2048].double()
        dg, du = dh * u * slope, dh * g * c
        dxs.append(dg @ wg + du @ wu)
        Gg += dg.T @ (x - mu)
        Gu += du.T @ (x - mu)
        sg += dg.sum(0)
        su += du.sum(0)
    out = [torch.cat(hs)]
    if kind == "train":
        out += [torch.cat(dxs), Gg, Gu] + ([sg, su] if case["bias"] else [])
    return out


def work(case):
    N, M, e = case["N"], case["M"], 2.0 if case["dtype"] == "bf16" else 4.0
    kind = case["kind"]
    if kind in ("norm", "norm8", "normgrad"):
        streams = {"norm": 2 * e, "norm8": e + 1, "normgrad": 3 * e}[kind]
        if case["residual"]:
            streams += e if kind == "normgrad" else 2 * e
        return {"bytes": N * M * streams + 4.0 * M * (2 if kind == "normgrad" else 1), "flops": N * M * (12.0 if kind == "normgrad" else 6.0)}
    S = case["S"]
    if kind == "int8":
        return {"bytes": N * M * (e if case["quantise"] else 1.0) + S * M + e * N * S, "flops": 2.0 * N * M * S}
    nbytes, flops = e * (N * M + 2.0 * S * M + N * S), 4.0 * N * M * S
    if kind == "train":
        nbytes, flops = nbytes + e * (N * S + N * M + 2.0 * S * M), 3 * flops
    return {"bytes": nbytes, "flops": flops}
