"""More layer operators of the library's denoisers: a linear layer with its epilogue, the norms before and after a
residual block fused with gate, residual scale and dropout, and dropout alone, each forward and as a training step.
Cases, inputs, plain forms, exact values and the work of a pass.

  linear          y = act(x W^T + b + table[step]) + residual; gradients of x, W, b and the table
  residual norm   q = post(h) (a norm with weight, or h itself), r' = r + alpha gate D q, n = (xhat(r') w + b) (1 + scale) + shift;
                  gate, scale and shift are one row per group of consecutive rows; gradients of all of them
  dropout         y = D x (+ residual); gradient D dy

  D: 0 or 1 / (1 - p), from Philox-4x32-10 with key `seed` and counter (column / 8, step, row, 3): eight columns share the
  four words of a block, 16 bits each, low half first; a column is dropped if its 16 bits are below round(65536 p), and
  1 / (1 - p) is that of the rounded p.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------


def _linear(name, op, rows, k, n, dtype, act, steps=0, residual=False, y=None):
    return dict(name=name, op=op, rows=rows, k=k, n=n, dtype=dtype, act=act, steps=steps, residual=residual, y=y or dtype)


def _norms(name, op, rows, d, r, h, kind, groups, mod, gate, weights, post, p):
    return dict(name=name, op=op, rows=rows, d=d, r=r, h=h, kind=kind, groups=groups, mod=mod, gate=gate, weights=weights,
                post=post, p=p)


def _dropout(name, op, rows, d, x, r, p):
    return dict(name=name, op=op, rows=rows, d=d, x=x, r=r, p=p)


def listed():
    return [
        # a hidden layer of the MLP denoiser for one chain at one position: the weights are read for a single row
        _linear("linear 1x2048x2048", "linear", 1, 2048, 2048, "bf16", "silu", steps=250),
        # the same layer in a batched target pass (2048 chains, windows of 8)
        _linear("linear 16384x2048x2048", "linear", 16384, 2048, 2048, "bf16", "silu", steps=250),
        # a count of outputs that nothing divides, the other 16-bit type
        _linear("linear 1037x1000x2731 f16", "linear", 1037, 1000, 2731, "f16", "gelu"),
        # the product that leads back to the float residual stream
        _linear("linear 16384x8192x2048 residual", "linear", 16384, 8192, 2048, "bf16", None, residual=True, y="f32"),
        # a training step on few rows
        _linear("linear train 256x1024x4096", "linear_train", 256, 1024, 4096, "bf16", "gelu_tanh"),
        # a training step of the hidden layer on a full batch, each row at its own step of the chain
        _linear("linear train 8192x2048x2048", "linear_train", 8192, 2048, 2048, "bf16", "silu", steps=250),
        # between two blocks for a few rows: latency
        _norms("norms 64x2048 rms", "norms", 64, 2048, "bf16", "bf16", "rms", 1, False, False, True, False, 0.0),
        # conditioned blocks: gate, scale and shift per sample of 256 rows, float stream
        _norms("norms 16384x2048 conditioned", "norms", 16384, 2048, "f32", "bf16", "layer", 64, True, True, False, False, 0.0),
        # training with norms on both sides of the block, a learned gate per channel and dropout
        _norms("norms train 16384x2048 sandwich", "norms_train", 16384, 2048, "f32", "bf16", "rms", 1, False, True, True, True, 0.1),
        # vector states: every row its own conditioning; odd width and odd count of rows, nothing is aligned
        _norms("norms train 1021x1001 f32", "norms_train", 1021, 1001, "f32", "f32", "layer", 1021, True, True, True, False, 0.0),
        # a small batch: latency
        _dropout("dropout 64x2048", "dropout", 64, 2048, "bf16", None, 0.1),
        # a block's output in training, added to the float stream, and its gradient
        _dropout("dropout train 16384x2048 residual", "dropout_train", 16384, 2048, "bf16", "f32", 0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear_train", "norms", "norms_train", "dropout", "dropout_train"])
    if op.startswith("linear"):
        k = 8 * _log_int(rng, 4, 1024)
        n = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            n = -(-n // 8) * 8
        most = 16384 * 8192 * 2048 if op == "linear" else 8192 * 2048 * 2048
        rows = max(1, min(_log_int(rng, 1, 16384), most // (k * n)))
        dtype = rng.choice(["bf16", "f16"])
        residual = rng.random() < 0.4
        return dict(op=op, rows=rows, k=k, n=n, dtype=dtype, act=rng.choice([None, "silu", "gelu", "gelu_tanh"]),
                    steps=rng.choice([0, 0, _log_int(rng, 1, 1000)]), residual=residual, y=rng.choice([dtype, "f32"]))
    d = _log_int(rng, 16, 16384)
    if rng.random() < 0.6:
        d = -(-d // 8) * 8
    rows = max(1, min(_log_int(rng, 1, 65536), 16384 * 2048 // d))
    p = rng.choice([0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)])
    if op.startswith("dropout"):
        x = rng.choice(["f32", "bf16", "f16"])
        return dict(op=op, rows=rows, d=d, x=x, r=rng.choice([None, x, "f32"]), p=p)
    r = rng.choice(["f32", "bf16", "f16"])
    h = rng.choice(["f32", "bf16", "f16"]) if r == "f32" else r
    groups = rng.choice([1, rows, _log_int(rng, 1, rows)])
    rows = rows // groups * groups
    return dict(op=op, rows=rows, d=d, r=r, h=h, kind=rng.choice(["layer", "rms"]), groups=groups, mod=rng.random() < 0.6,
                gate=rng.random() < 0.6, weights=rng.random() < 0.6, post=rng.random() < 0.4, p=p)


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _linear_inputs(case, seed):
    g = _gen(seed)
    rows, k, n, t = case["rows"], case["k"], case["n"], TYPES[case["dtype"]]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(x=rnd(rows, k).to(t), w=(rnd(n, k) * k ** -0.5).to(t), b=0.2 * rnd(n), table=None, step=None, residual=None)
    if case["steps"]:
        s["table"] = (0.5 * rnd(case["steps"], n)).to(t)
        s["step"] = torch.randint(0, case["steps"], (rows,), generator=g, device="cuda", dtype=torch.int32)
    if case["residual"]:
        s["residual"] = rnd(rows, n).to(TYPES[case["y"]])
    if case["op"] == "linear_train":
        s["dy"] = (rnd(rows, n) * 0.0625).to(TYPES[case["y"]])
    return s


def _norms_inputs(case, seed):
    g = _gen(seed)
    rows, d, groups = case["rows"], case["d"], case["groups"]
    tr, th = TYPES[case["r"]], TYPES[case["h"]]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # a residual stream: rows of different scale and offset, some channels much larger than the others
    r = rnd(rows, d)
    r *= torch.exp(0.5 * rnd(rows, 1))
    r *= 1.0 + 7.0 * (torch.rand(d, generator=g, device="cuda") < 0.02)
    r += rnd(rows, 1)
    s = dict(r=r.to(tr), h=rnd(rows, d).to(th), seed=int(seed) & 0x7FFFFFFF, alpha=0.7071)
    # conditioning comes as one product's columns: slices of one tensor
    cond = (0.3 * rnd(groups, 3 * d)).to(th)
    s["gate"] = cond[:, :d] if case["gate"] else None
    s["scale"], s["shift"] = (cond[:, d:2 * d], cond[:, 2 * d:]) if case["mod"] else (None, None)
    s["w"], s["b"] = (1.0 + 0.2 * rnd(d), 0.2 * rnd(d)) if case["weights"] else (None, None)
    s["wp"] = 1.0 + 0.2 * rnd(d) if case["post"] else None
    if case["op"] == "norms_train":
        s["dn"], s["dr"] = (0.1 * rnd(rows, d)).to(th), (0.1 * rnd(rows, d)).to(tr)
    return s


def _dropout_inputs(case, seed):
    g = _gen(seed)
    rows, d = case["rows"], case["d"]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(x=rnd(rows, d).to(TYPES[case["x"]]), seed=int(seed) & 0x7FFFFFFF, residual=None)
    if case["r"]:
        s["residual"] = rnd(rows, d).to(TYPES[case["r"]])
    if case["op"] == "dropout_train":
        s["dy"] = rnd(rows, d).to(TYPES[case["r"] or case["x"]])
    return s


def prepare(case, seed):
    make = _linear_inputs if case["op"].startswith("linear") else _norms_inputs if case["op"].startswith("norms") else _dropout_inputs
    s = make(case, seed)
    s["case"] = case
    return s


STEP = 17                                                # of the generator's counter: the training step


# ---------------------------------------------------------------------------------------------
# one pass: plain forms in 32 bits, rounded once at the end, or the library's calls
# ---------------------------------------------------------------------------------------------


def _plain_factor(rows, d, p, seed):
    """D [rows, d] in float, from the generator in 64-bit integers."""
    m32 = 0xFFFFFFFF
    nb = (d + 7) // 8
    c0 = torch.arange(nb, device="cuda").expand(rows, nb)
    c2 = torch.arange(rows, device="cuda")[:, None].expand(rows, nb)
    c1, c3 = torch.full_like(c0, STEP), torch.full_like(c0, 3)
    k0, k1 = seed & m32, (seed >> 32) & m32
    for _ in range(10):
        # (the low 64 bits of the product are right even where it passes the sign bit)
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & m32) ^ c1 ^ k0, b & m32, ((a >> 32) & m32) ^ c3 ^ k1, a & m32
        k0, k1 = (k0 + 0x9E3779B9) & m32, (k1 + 0xBB67AE85) & m32
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    draws = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, nb * 8)[:, :d]
    thr = round(p * 65536)
    return (draws >= thr).float() * (65536.0 / (65536 - thr))


def _plain_act(g, act):
    """act(g) and its derivative."""
    if act is None:
        return g, torch.ones_like(g)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    k, c = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(k * (g + c * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3.0 * c * g * g)


def _plain_linear(s, train):
    case = s["case"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["b"]
    if s["table"] is not None:
        z = z + s["table"].float()[s["step"].long()]
    a, da = _plain_act(z, case["act"])
    y = a if s["residual"] is None else a + s["residual"].float()
    y = y.to(TYPES[case["y"]])
    if not train:
        return y
    dz = s["dy"].float() * da
    dx, dw = (dz @ w).to(s["x"].dtype), (dz.t() @ x).to(s["w"].dtype)
    db = dz.double().sum(dim=0).float()
    if s["table"] is None:
        return y, dx, dw, db
    rows_of_step = (torch.arange(case["steps"], device="cuda")[:, None] == s["step"]).float()
    return y, dx, dw, db, (rows_of_step @ dz).to(s["table"].dtype)


def _plain_xhat(v, kind):
    """The normalised rows and 1 / their size."""
    if kind == "layer":
        # (the mean in 64 bits: rows may sit far from zero, and what is left after it is what counts)
        v = (v.double() - v.double().mean(dim=1, keepdim=True)).float()
    rstd = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * rstd, rstd


def _plain_xhat_gradient(d, xhat, rstd, kind):
    c = xhat * (d * xhat).mean(dim=1, keepdim=True)
    if kind == "layer":
        c = c + d.mean(dim=1, keepdim=True)
    return (d - c) * rstd


def _plain_norms(s, train):
    case = s["case"]
    rows, d, groups, kind = case["rows"], case["d"], case["groups"], case["kind"]
    per = rows // groups
    spread = lambda v: v.float().repeat_interleave(per, dim=0)  # noqa: E731
    r, h = s["r"].float(), s["h"].float()
    w = s["w"] if s["w"] is not None else torch.ones(d, device="cuda")
    b = s["b"] if s["b"] is not None else torch.zeros(d, device="cuda")
    gate = spread(s["gate"]) if s["gate"] is not None else torch.ones(1, device="cuda")
    scale = 1.0 + spread(s["scale"]) if s["scale"] is not None else torch.ones(1, device="cuda")
    shift = spread(s["shift"]) if s["shift"] is not None else torch.zeros(1, device="cuda")
    phat, prstd = _plain_xhat(h, kind) if case["post"] else (h, None)
    q = phat * s["wp"] if case["post"] else h
    keep = _plain_factor(rows, d, case["p"], s["seed"]) if case["p"] else torch.ones(1, device="cuda")
    out = r + s["alpha"] * gate * (keep * q)
    xhat, rstd = _plain_xhat(out, kind)
    u = xhat * w + b
    n = (u * scale + shift).to(s["h"].dtype)
    if not train:
        return out.to(s["r"].dtype), n
    dn, dr = s["dn"].float(), s["dr"].float()
    sums = lambda v: v.reshape(groups, per, d).sum(dim=1)  # noqa: E731
    du = dn * scale
    g = dr + _plain_xhat_gradient(du * w, xhat, rstd, kind)
    dq = s["alpha"] * gate * keep * g
    res = [out.to(s["r"].dtype), n, g.to(s["r"].dtype)]
    res.append((_plain_xhat_gradient(dq * s["wp"], phat, prstd, kind) if case["post"] else dq).to(s["h"].dtype))
    if case["weights"]:
        res += [(du * xhat).sum(dim=0), du.sum(dim=0)]
    if case["mod"]:
        res += [sums(dn * u).to(s["scale"].dtype), sums(dn).to(s["shift"].dtype)]
    if case["gate"]:
        res.append(sums(s["alpha"] * g * (keep * q)).to(s["gate"].dtype))
    if case["post"]:
        res.append((dq * phat).sum(dim=0))
    return tuple(res)


def _plain_dropout(s, train):
    case = s["case"]
    keep = _plain_factor(case["rows"], case["d"], case["p"], s["seed"])
    y = keep * s["x"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(TYPES[case["r"] or case["x"]])
    return (y, (keep * s["dy"].float()).to(s["x"].dtype)) if train else y


def _own_linear(s, train):
    import paper_2501_05370_b200 as sds
    case = s["case"]
    kw = dict(table=s["table"], step=s["step"], residual=s["residual"], out_dtype=TYPES[case["y"]])
    if not train:
        return sds.linear(s["x"], s["w"], s["b"], case["act"], **kw)
    y, kept = sds.linear(s["x"], s["w"], s["b"], case["act"], keep=True, **kw)
    dx, dw, db, dtable = sds.linear_backward(s["dy"], s["x"], s["w"], kept, bias=s["b"], table=s["table"], step=s["step"])
    return (y, dx, dw, db) if dtable is None else (y, dx, dw, db, dtable)


def _own_norms(s, train):
    import paper_2501_05370_b200 as sds
    case = s["case"]
    kw = dict(weight=s["w"], bias=s["b"], scale=s["scale"], shift=s["shift"], gate=s["gate"], post=case["post"],
              post_weight=s["wp"], kind=case["kind"], alpha=s["alpha"], p=case["p"], seed=s["seed"], step=STEP)
    if not train:
        return sds.residual_norm(s["r"], s["h"], eps=EPS, **kw)
    r, n, kept = sds.residual_norm(s["r"], s["h"], eps=EPS, keep=True, **kw)
    grads = sds.residual_norm_backward(s["dn"], s["dr"], s["r"], s["h"], kept, **kw)
    return (r, n, *[g for g in grads if g is not None])


def _own_dropout(s, train):
    import paper_2501_05370_b200 as sds
    p, seed = s["case"]["p"], s["seed"]
    y = sds.dropout(s["x"], p, seed, STEP, residual=s["residual"])
    return (y, sds.dropout_backward(s["dy"], p, seed, STEP, out_dtype=s["x"].dtype)) if train else y


def run(state):
    op = state["case"]["op"]
    train = op.endswith("_train")
    if op.startswith("linear"):
        return _own_linear(state, train) if own else _plain_linear(state, train)
    if op.startswith("norms"):
        return _own_norms(state, train) if own else _plain_norms(state, train)
    return _own_dropout(state, train) if own else _plain_dropout(state, train)


# ---------------------------------------------------------------------------------------------
# work of a pass, and its exact values
# ---------------------------------------------------------------------------------------------


def work(case):
    size = lambda t: TYPES[t].itemsize  # noqa: E731
    op, rows = case["op"], case["rows"]
    if op.startswith("linear"):
        k, n, sz, sy = case["k"], case["n"], size(case["dtype"]), size(case["y"])
        table = case["steps"] * n * sz
        fixed = sz * n * k + 4 * n + table + (4 * rows if case["steps"] else 0)
        bytes_ = sz * rows * k + sy * rows * n * (2 if case["residual"] else 1) + fixed
        if op == "linear":
            return {"bytes": bytes_, "flops": 2 * rows * k * n}
        # dy in, dx, dW, db and the table's gradient out
        return {"bytes": bytes_ + sy * rows * n + sz * rows * k + sz * n * k + 4 * n + table, "flops": 6 * rows * k * n}
    d = case["d"]
    e = rows * d
    if op.startswith("dropout"):
        sx, sr = size(case["x"]), size(case["r"] or case["x"])
        bytes_ = e * (sx + sr + (sr if case["r"] else 0))
        return {"bytes": bytes_ + (e * (sx + sr) if op == "dropout_train" else 0), "flops": (3 if op == "dropout" else 4) * e}
    sr, sh = size(case["r"]), size(case["h"])
    cond = case["groups"] * d * sh * ((1 if case["gate"] else 0) + (2 if case["mod"] else 0))
    vectors = 4 * d * ((2 if case["weights"] else 0) + (1 if case["post"] else 0))
    if op == "norms":
        return {"bytes": 2 * e * (sr + sh) + cond + vectors, "flops": 12 * e}
    # r, h, dn and dr in; r', n and the gradients of r and h out; conditioning and weights in, their gradients out
    return {"bytes": 4 * e * (sr + sh) + 2 * (cond + vectors), "flops": 40 * e}


def _exact_factor(rows, d, p, seed):
    """D in 64 bits: the generator on the host, in numpy's unsigned integers, row by row of counters."""
    thr = round(p * 65536)
    blocks = -(-d // 8)
    ctr = np.empty((4, rows * blocks), np.uint32)
    ctr[0] = np.tile(np.arange(blocks, dtype=np.uint32), rows)
    ctr[1] = STEP
    ctr[2] = np.repeat(np.arange(rows, dtype=np.uint32), blocks)
    ctr[3] = 3
    key = [np.uint32(seed & 0xFFFFFFFF), np.uint32(seed >> 32)]
    for i in range(10):
        even = np.uint64(0xD2511F53) * ctr[0].astype(np.uint64)
        odd = np.uint64(0xCD9E8D57) * ctr[2].astype(np.uint64)
        left = (odd >> np.uint64(32)).astype(np.uint32) ^ ctr[1] ^ key[0]
        right = (even >> np.uint64(32)).astype(np.uint32) ^ ctr[3] ^ key[1]
        ctr = np.stack([left, odd.astype(np.uint32), right, even.astype(np.uint32)])
        key = [np.uint32((int(key[0]) + 0x9E3779B9) % 2 ** 32), np.uint32((int(key[1]) + 0xBB67AE85) % 2 ** 32)]
    halves = np.ascontiguousarray(ctr.T).view("<u2").reshape(rows, blocks * 8)[:, :d]
    keep = torch.from_numpy(halves >= thr).to("cuda")
    return keep.double() / (1.0 - thr / 65536.0)


def _exact_linear(s, train):
    case = s["case"]
    v = {n: s[n].double().requires_grad_(train) for n in ("x", "w", "b", "table") if s[n] is not None}
    z = torch.mm(v["x"], v["w"].T).add(v["b"])
    if "table" in v:
        z = z + torch.index_select(v["table"], 0, s["step"].long())
    if case["act"] == "silu":
        z = z * torch.sigmoid(z)
    elif case["act"] == "gelu":
        z = z * (1.0 - 0.5 * torch.erfc(z / math.sqrt(2.0)))
    elif case["act"] == "gelu_tanh":
        z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3)))
    y = z if s["residual"] is None else z + s["residual"].double()
    if not train:
        return y.detach()
    return (y.detach(), *torch.autograd.grad(y, list(v.values()), s["dy"].double()))


def _exact_norms(s, train):
    case = s["case"]
    rows, d, groups = case["rows"], case["d"], case["groups"]
    names = ["r", "h"] + (["w", "b"] if case["weights"] else []) + (["scale", "shift"] if case["mod"] else [])
    names += (["gate"] if case["gate"] else []) + (["wp"] if case["post"] else [])
    v = {n: s[n].double().requires_grad_(train) for n in names}

    def norm(t):
        if case["kind"] == "layer":
            t = t - t.sum(dim=-1, keepdim=True) / d
        return t / torch.sqrt(t.pow(2).sum(dim=-1, keepdim=True) / d + EPS)

    grouped = lambda t: t.view(groups, rows // groups, d)  # noqa: E731
    branch = norm(v["h"]) * v["wp"] if case["post"] else v["h"]
    if case["p"]:
        branch = branch * _exact_factor(rows, d, case["p"], s["seed"])
    branch = s["alpha"] * grouped(branch)
    if case["gate"]:
        branch = branch * v["gate"][:, None, :]
    out = grouped(v["r"]) + branch
    n = norm(out)
    if case["weights"]:
        n = n * v["w"] + v["b"]
    if case["mod"]:
        n = n * (1.0 + v["scale"][:, None, :]) + v["shift"][:, None, :]
    out, n = out.view(rows, d), n.reshape(rows, d)
    if not train:
        return out.detach(), n.detach()
    grads = torch.autograd.grad([out, n], list(v.values()), [s["dr"].double(), s["dn"].double()])
    return (out.detach(), n.detach(), *grads)


def exact(case, seed):
    """The definitions in 64 bits; the gradients by differentiating them."""
    s = prepare(case, seed)
    train = case["op"].endswith("_train")
    if case["op"].startswith("linear"):
        return _exact_linear(s, train)
    if case["op"].startswith("norms"):
        return _exact_norms(s, train)
    keep = _exact_factor(case["rows"], case["d"], case["p"], s["seed"])
    y = keep * s["x"].double()
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return (y, keep * s["dy"].double()) if train else y
