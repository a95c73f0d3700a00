"""The layer operators of the library's gated denoisers: layer norm and the gated feed-forward block, each
forward and as a training step. Cases, inputs, plain forms, exact values and the work of a pass.

  layer norm          y = (x - mean) / sqrt(var + eps) * w + b over the last axis;
                      gradients dx, dw = sum_rows dy * xhat, db = sum_rows dy
  gated feed-forward  y = (act(x Wg^T) * (x Wu^T)) Wd^T with Wg, Wu [f, d] and Wd [d, f];
                      gradients of x and of the three weights
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------


def _norm(name, op, rows, d, x, y):
    return dict(name=name, op=op, rows=rows, d=d, x=x, y=y)


def _ffn(name, op, rows, d, f, dtype, act):
    return dict(name=name, op=op, rows=rows, d=d, f=f, dtype=dtype, act=act)


def listed():
    return [
        # the rows of one target pass of a small batch of chains: latency of a launch
        _norm("norm 64x2048", "norm", 64, 2048, "bf16", "bf16"),
        # a batched target pass (2048 chains, windows of 8): the float residual stream in, 16-bit rows out
        _norm("norm 16384x2048 mixed", "norm", 16384, 2048, "f32", "bf16"),
        # long states in float, a count of rows that no tile divides
        _norm("norm 2047x16384 f32", "norm", 2047, 16384, "f32", "f32"),
        # training a denoiser of that width: statistics kept, weight gradients over all rows
        _norm("norm train 16384x2048", "norm_train", 16384, 2048, "bf16", "bf16"),
        # odd width and odd count of rows: nothing is aligned
        _norm("norm train 1021x1001 f32", "norm_train", 1021, 1001, "f32", "f32"),
        # few long rows: the weight gradients have as many columns as there is memory traffic
        _norm("norm train 512x16384 mixed", "norm_train", 512, 16384, "f32", "bf16"),
        # one chain, one position: the weights are read for a single row
        _ffn("ffn 1x2048x8192", "ffn", 1, 2048, 8192, "bf16", "silu"),
        # 64 chains, one position each, in the other 16-bit type and activation
        _ffn("ffn 64x2048x8192 f16", "ffn", 64, 2048, 8192, "f16", "gelu"),
        # a batched target pass (2048 chains, windows of 8)
        _ffn("ffn 16384x2048x8192", "ffn", 16384, 2048, 8192, "bf16", "silu"),
        # a training step on few rows
        _ffn("ffn train 256x1024x4096", "ffn_train", 256, 1024, 4096, "bf16", "silu"),
        # sizes that no tile divides
        _ffn("ffn train 1037x1000x2728 f16", "ffn_train", 1037, 1000, 2728, "f16", "gelu_tanh"),
        # a training step on a full batch
        _ffn("ffn train 8192x2048x8192", "ffn_train", 8192, 2048, 8192, "bf16", "silu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_train", "ffn", "ffn_train"])
    if op.startswith("norm"):
        d = _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            d = -(-d // 8) * 8
        rows = max(1, min(_log_int(rng, 1, 65536), 16384 * 2048 // d))
        x = rng.choice(["f32", "bf16", "f16"])
        y = rng.choice(["f32", "bf16", "f16"]) if x == "f32" else x
        return dict(op=op, rows=rows, d=d, x=x, y=y)
    d = 8 * _log_int(rng, 8, 512)
    f = 8 * _log_int(rng, 16, 1536)
    most = 16384 * 2048 * 8192 if op == "ffn" else 8192 * 2048 * 8192
    rows = max(1, min(_log_int(rng, 1, 16384), most // (d * f)))
    return dict(op=op, rows=rows, d=d, f=f, dtype=rng.choice(["bf16", "f16"]),
                act=rng.choice(["silu", "gelu", "gelu_tanh"]))


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _norm_inputs(case, seed):
    g = _gen(seed)
    rows, d = case["rows"], case["d"]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # a residual stream: rows of different scale and offset, some channels much larger than the others
    x = rnd(rows, d)
    x *= torch.exp(0.5 * rnd(rows, 1))
    x *= 1.0 + 7.0 * (torch.rand(d, generator=g, device="cuda") < 0.02)
    x += rnd(rows, 1)
    s = dict(x=x.to(TYPES[case["x"]]), w=1.0 + 0.2 * rnd(d), b=0.2 * rnd(d))
    if case["op"] == "norm_train":
        s["dy"] = (rnd(rows, d) * 0.1).to(TYPES[case["y"]])
    return s


def _ffn_inputs(case, seed):
    g = _gen(seed)
    rows, d, f, t = case["rows"], case["d"], case["f"], TYPES[case["dtype"]]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(x=rnd(rows, d).to(t), wg=(rnd(f, d) * d ** -0.5).to(t), wu=(rnd(f, d) * d ** -0.5).to(t),
             wd=(rnd(d, f) * f ** -0.5).to(t))
    if case["op"] == "ffn_train":
        s["dy"] = (rnd(rows, d) * 0.0625).to(t)
    return s


def prepare(case, seed):
    s = _norm_inputs(case, seed) if case["op"].startswith("norm") else _ffn_inputs(case, seed)
    s["case"] = case
    return s


# ---------------------------------------------------------------------------------------------
# one pass: plain forms in 32 bits, rounded once at the end, or the library's calls
# ---------------------------------------------------------------------------------------------


def _plain_norm(s, train):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    t = TYPES[s["case"]["y"]]
    # (the mean in 64 bits: rows may sit far from zero, and what is left after it is what counts)
    mean = x.double().mean(dim=1, keepdim=True)
    xc = (x.double() - mean).float()
    rstd = torch.rsqrt((xc * xc).mean(dim=1, keepdim=True) + EPS)
    xhat = xc * rstd
    y = (xhat * w + b).to(t)
    if not train:
        return y
    dy = s["dy"].float()
    wdy = dy * w
    c1 = wdy.mean(dim=1, keepdim=True)
    c2 = (wdy * xhat).mean(dim=1, keepdim=True)
    dx = ((wdy - c1 - xhat * c2) * rstd).to(s["x"].dtype)
    dw = (dy * xhat).sum(dim=0)
    db = dy.sum(dim=0)
    return y, dx, dw, db


def _plain_act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    k, c = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(k * (g + c * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3.0 * c * g * g)


def _plain_ffn(s, train):
    act, t = s["case"]["act"], s["x"].dtype
    x, wg, wu, wd = s["x"].float(), s["wg"].float(), s["wu"].float(), s["wd"].float()
    g = x @ wg.t()
    u = x @ wu.t()
    a, da = _plain_act(g, act)
    h = a * u
    y = (h @ wd.t()).to(t)
    if not train:
        return y
    dy = s["dy"].float()
    dh = dy @ wd
    dwd = (dy.t() @ h).to(t)
    dg = dh * u * da
    du = dh * a
    dx = (dg @ wg + du @ wu).to(t)
    return y, dx, (dg.t() @ x).to(t), (du.t() @ x).to(t), dwd


def _own_norm(s, train):
    import paper_2501_05370_b200 as sds
    t = TYPES[s["case"]["y"]]
    if not train:
        return sds.layer_norm(s["x"], s["w"], s["b"], EPS, out_dtype=t)
    y, mean, rstd = sds.layer_norm(s["x"], s["w"], s["b"], EPS, out_dtype=t, stats=True)
    dx, dw, db = sds.layer_norm_backward(s["dy"], s["x"], s["w"], mean, rstd)
    return y, dx, dw, db


def _own_ffn(s, train):
    import paper_2501_05370_b200 as sds
    act = s["case"]["act"]
    if not train:
        return sds.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], act)
    y, kept = sds.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], act, keep=True)
    dx, dwg, dwu, dwd = sds.gated_ffn_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], kept)
    return y, dx, dwg, dwu, dwd


def run(state):
    op = state["case"]["op"]
    train = op.endswith("_train")
    if op.startswith("norm"):
        return _own_norm(state, train) if own else _plain_norm(state, train)
    return _own_ffn(state, train) if own else _plain_ffn(state, train)


# ---------------------------------------------------------------------------------------------
# work of a pass, and its exact values
# ---------------------------------------------------------------------------------------------


def work(case):
    size = lambda t: TYPES[t].itemsize  # noqa: E731
    rows, d = case["rows"], case["d"]
    if case["op"].startswith("norm"):
        n, sx, sy = rows * d, size(case["x"]), size(case["y"])
        if case["op"] == "norm":
            return {"bytes": n * (sx + sy) + 8 * d, "flops": 8 * n}
        # x and dy in; y, dx and the two weight gradients out
        return {"bytes": n * (2 * sx + 2 * sy) + 16 * d, "flops": 24 * n}
    f, sz = case["f"], size(case["dtype"])
    if case["op"] == "ffn":
        return {"bytes": sz * (2 * rows * d + 3 * d * f), "flops": 6 * rows * d * f}
    # x and dy in, y and dx out; the weights in, their gradients out
    return {"bytes": sz * (4 * rows * d + 6 * d * f), "flops": 18 * rows * d * f}


def exact(case, seed):
    """The definitions in 64 bits; the gradients by differentiating them."""
    s = prepare(case, seed)
    train = case["op"].endswith("_train")
    names = ["x", "w", "b"] if case["op"].startswith("norm") else ["x", "wg", "wu", "wd"]
    v = {n: s[n].double().requires_grad_(train) for n in names}
    if case["op"].startswith("norm"):
        centred = v["x"] - v["x"].sum(dim=1, keepdim=True) / case["d"]
        var = centred.pow(2).sum(dim=1, keepdim=True) / case["d"]
        y = v["w"] * (centred / torch.sqrt(var + EPS)) + v["b"]
    else:
        gate, up = torch.mm(v["x"], v["wg"].T), torch.mm(v["x"], v["wu"].T)
        if case["act"] == "silu":
            gate = gate * torch.sigmoid(gate)
        elif case["act"] == "gelu":
            gate = gate * (1.0 - 0.5 * torch.erfc(gate / math.sqrt(2.0)))
        else:
            gate = gate * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate.pow(3)))
        y = torch.mm(gate * up, v["wd"].T)
    if not train:
        return y.detach()
    grads = torch.autograd.grad(y, [v[n] for n in names], s["dy"].double())
    return (y.detach(), *grads)
