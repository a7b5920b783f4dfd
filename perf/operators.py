"""Timed calls of the operators on both sides of the compressor step: the matrix product with bias, activation, dropout
and residual that reads a plan's parameters, its backward pass that writes a plan's gradients, dropout by itself, and the
compressor that keeps a random subset of the update.  All of them draw from one counter-based generator, so no mask is
stored anywhere.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a training or serving program holds
before the call, run() is one call, work() the bytes and operations it cannot do without, exact() the same outputs in 64 bits.

The generator is Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011):
four 32-bit words from a 128-bit counter and a 64-bit key.  The key is the seed.  Dropout of element (row, col): the
counter is (col / 8, row, offset), the eight 16-bit halves of the words (low half first) belong to the eight columns, and
an element is dropped where its half is below round(65536 p).  Random mask of entry `pos` of the flattened matrix of
tensor t: the counter is (pos / 4, t, offset), word pos % 4, kept where it is below the threshold.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
MOST = {"f32": 6.0e10, "bf16": 1.7e12}   # operations of one product


def _linear(name, pass_, tokens, n, k, dtype, act="identity", drop=0.0, residual=False, pre=False, params=None, pad=0):
    return dict(name=name, op="linear", dir=pass_, tokens=tokens, n=n, k=k, dtype=dtype, act=act, drop=drop,
                residual=residual, pre=pre, params=params or dtype, pad=pad)


def _dropout(name, pass_, rows, cols, dtype, drop, residual=False, pad=0):
    return dict(name=name, op="dropout", dir=pass_, rows=rows, cols=cols, dtype=dtype, drop=drop, residual=residual, pad=pad)


def _mask(name, family, dtype, workers, keep, **size):
    return dict(name=name, op="mask", family=family, dtype=dtype, workers=workers, keep=keep, **size)


def listed():
    return [
        # one new token through the first feed-forward matrix of a transformer layer: the weights are read, nothing else counts
        _linear("token_ff1_bf16", "forward", 1, 8192, 2048, "bf16", act="gelu"),
        # nineteen sequences' next tokens through the second one, residual added, from the fp32 parameters that the update steps
        _linear("tokens19_ff2_bf16", "forward", 19, 2048, 8192, "bf16", residual=True, params="f32"),
        # training: the first feed-forward matrix over a batch of 4096 tokens, what enters the activation kept for the backward pass
        _linear("ff1_bf16", "forward", 4096, 8192, 2048, "bf16", act="gelu", pre=True),
        # training: the second one over a ragged batch, dropout and residual behind it
        _linear("ff2_dropout_bf16", "forward", 4099, 2048, 8192, "bf16", drop=0.1, residual=True),
        # its backward pass through dropout and activation, weights as the update's fp32 parameters
        _linear("ff1_backward_bf16", "backward", 4096, 8192, 2048, "bf16", act="gelu", drop=0.1, params="f32"),
        # logits of a long batch over the whole vocabulary: the largest product
        _linear("vocabulary_bf16", "forward", 8192, 50304, 2048, "bf16"),
        # the gates of an LSTM language model, 20 sequences of 35 steps, rows of 650 (not a multiple of four)
        _linear("lstm_gates_backward_f32", "backward", 700, 2600, 650, "f32"),
        # dropout between that model's layers: a small call, where latency counts
        _dropout("lstm_dropout_f32", "forward", 700, 650, "f32", 0.5),
        # dropout and residual of a transformer's attention projection over a long batch
        _dropout("residual_dropout_bf16", "forward", 16384, 2048, "bf16", 0.1, residual=True),
        # gradient of dropout behind a wide activation, odd row length
        _dropout("wide_dropout_backward_bf16", "backward", 8191, 8191, "bf16", 0.1),
        # compression of every gradient matrix of a ResNet18 with PowerSGD's budget at rank 2, sixteen workers
        _mask("random_mask_resnet18_w16", "resnet18", "f32", 16, -1.0, width=64),
        # four layers and the embedding of a transformer, bf16 gradients, one entry in a hundred kept
        _mask("random_mask_transformer4", "transformer", "bf16", 1, 0.01, layers=4, d=2048, vocab=50304),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator at sizes between its smallest sensible ones and the listed ones."""
    op = rng.choice(["linear", "linear", "linear", "linear", "dropout", "mask"])
    drop = rng.choice([0.0, 0.1, 0.2, 0.5])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "dropout":
        while True:
            rows, cols = _log(rng, 1, 16384), _log(rng, 16, 16384)
            if rows * cols <= 8191 * 8191:
                break
        back = rng.random() < 0.5
        c = _dropout("", "backward" if back else "forward", rows, cols, dtype, drop or 0.3, residual=not back and rng.random() < 0.5,
                     pad=rng.choice([0, 0, 8, 5]))
    elif op == "mask":
        workers, keep = rng.choice([1, 1, 2, 3, 4, 8, 16]), rng.choice([-1.0, -1.0, 0.3, 0.05, 0.001])
        if rng.random() < 0.6:
            c = _mask("", "resnet18", dtype, workers, keep, width=rng.randrange(16, 65))
        else:
            c = _mask("", "transformer", dtype, rng.choice([1, 1, 2]), keep, layers=rng.randrange(1, 5), d=4 * _log(rng, 64, 256),
                      vocab=4 * _log(rng, 500, 12576))
    else:
        unit = rng.choice([1, 1, 8, 64])
        while True:
            tokens = _log(rng, 1, 8192)
            n, k = unit * max(1, _log(rng, 16, 50304) // unit), unit * max(1, _log(rng, 16, 8192) // unit)
            if k >= 2 and 2.0 * tokens * n * k <= MOST[dtype]:
                break
        act = rng.choice(["identity", "identity", "relu", "gelu", "gelu_tanh", "silu"])
        if rng.random() < 0.4:
            c = _linear("", "backward", tokens, n, k, dtype, act=act, drop=drop, params=rng.choice([dtype, "f32"]))
        else:
            c = _linear("", "forward", tokens, n, k, dtype, act=act, drop=drop, residual=rng.random() < 0.5,
                        pre=act != "identity" and rng.random() < 0.5, params=rng.choice([dtype, dtype, "f32"]), pad=rng.choice([0, 0, 8, 5]))
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------

def mask_shapes(case):
    """The gradient matrices (and vectors) of the model, as a plan is given them."""
    shapes = []
    if case["family"] == "resnet18":   # layer widths scale with the first one
        w = case["width"]
        shapes += [(w, 27), (w,), (w,)]
        for cin, c, first in ((w, w, 0), (w, 2 * w, 1), (2 * w, 4 * w, 1), (4 * w, 8 * w, 1)):
            shapes += [(c, 9 * cin), (c,), (c,), (c, 9 * c), (c,), (c,)]
            if first:
                shapes += [(c, cin), (c,), (c,)]
            shapes += [(c, 9 * c), (c,), (c,)] * 2
        return shapes + [(10, 8 * w), (10,)]
    d = case["d"]
    shapes.append((case["vocab"], d))
    for _ in range(case["layers"]):
        shapes += [(d, d), (d,)] * 4 + [(4 * d, d), (4 * d,), (d, 4 * d), (d,)] + [(d,)] * 4
    return shapes + [(d,)] * 2


def _up(a, b):
    return (a + b - 1) // b * b


def placed(shapes):
    """Offsets of the tensors in a plan's flat layout, its matrix elements N and its vector elements L."""
    n = sum(_up(math.prod(s), 64) for s in shapes if len(s) == 2)
    at, vec, off = 0, n, []
    for s in shapes:
        if len(s) == 2:
            off.append(at)
            at += _up(math.prod(s), 64)
        else:
            off.append(vec)
            vec += s[0]
    return off, n, vec - n


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DT[case["dtype"]]

    def normal(*size, dtype=dt, std=1.0, pad=0):
        if pad:
            return (torch.randn(size[0], size[1] + pad, generator=gen, device=dev) * std).to(dtype)[:, :size[1]]
        return (torch.randn(*size, generator=gen, device=dev) * std).to(dtype)

    s = dict(case=case, stream=torch.cuda.current_stream(dev).cuda_stream,
             rng=torch.tensor([0x9E3779B97F4A7C15 * (seed + 1) % (1 << 63), 1000 + seed], dtype=torch.int64, device=dev))
    if case["op"] == "linear":
        T, n, k = case["tokens"], case["n"], case["k"]
        shapes = [(n, k), (n,)]
        off, N, L = placed(shapes)
        # parameters and gradients in the plan's layout: weights of a trained layer's size, a small bias
        param = torch.zeros(N + L, dtype=DT[case["params"]], device=dev)
        param[:n * k] = normal(n * k, dtype=param.dtype, std=1.0 / math.sqrt(k))
        param[N:] = normal(n, dtype=param.dtype, std=0.1)
        s.update(param=param, x=normal(T, k, pad=case["pad"]))
        if case["dir"] == "forward":
            s["y"] = torch.zeros(T, n, dtype=dt, device=dev)
            s["residual"] = normal(T, n, pad=case["pad"]) if case["residual"] else None
            s["pre"] = torch.zeros(T, n, dtype=dt, device=dev) if case["pre"] else None
        else:
            s["dy"] = normal(T, n, std=1.0 / T, pad=case["pad"])
            s["pre"] = normal(T, n) if case["act"] != "identity" else None
            s["dx"] = torch.zeros(T, k, dtype=dt, device=dev)
            s["grad"] = torch.zeros(_up(N + L, 64), dtype=dt, device=dev)
    elif case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["cols"], pad=case["pad"])
        s["residual"] = normal(case["rows"], case["cols"], pad=case["pad"]) if case["residual"] else None
        s["y"] = torch.zeros(case["rows"], case["cols"], dtype=dt, device=dev)
    else:
        # gradients of noise around a shared part, and the error memory that earlier steps left: noise of the gradient's size
        shapes, W = mask_shapes(case), case["workers"]
        off, N, L = placed(shapes)
        stride = _up(N + L, 64)
        base = normal(stride, dtype=torch.float32, std=0.02)
        s["grad"] = torch.empty(W, stride, dtype=dt, device=dev)
        s["err"] = torch.empty(W, N, dtype=torch.float32, device=dev)
        for w in range(W):
            s["grad"][w] = (base + normal(stride, dtype=torch.float32, std=0.01)).to(dt)
            s["err"][w] = normal(N, dtype=torch.float32, std=0.03)
        s["out"] = torch.zeros(N + L, dtype=dt, device=dev)
    if own:
        from paper_1905_13727_amd import binding as B
        if case["op"] != "dropout":
            code = {"f32": B.PSGD_F32, "bf16": B.PSGD_BF16}
            s["plan"] = B.Plan(shapes, 2, case.get("workers", 1), code[case["dtype"]], code[case["dtype"]])
            if case["op"] == "mask":
                s["plan"].check(s["stream"])   # the plan's tables go to the device here, once
            else:
                size = s["plan"].linear_workspace(0, T, code[case["params"]])
                s["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=dev)
    return s


# ---- the plain form: elementary torch operations in 32 bits ----------------------------------------------------------

M32 = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, rng):
    """Four words (int64 tensors of 32-bit values) of the counters, which broadcast; the key is rng[0]."""
    k0, k1 = rng[0] & M32, (rng[0] >> 32) & M32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57   # 64-bit products, kept modulo 2^64
        c0, c1, c2, c3 = ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c0, c1, c2, c3


def _dropped(rows, cols, p, rng):
    """Truth values [rows, cols] of dropped elements, and the factor of the others."""
    d = int(math.floor(p * 65536 + 0.5))
    c0 = torch.arange((cols + 7) // 8, device=rng.device).view(1, -1)
    c1 = torch.arange(rows, device=rng.device).view(-1, 1)
    words = torch.stack(torch.broadcast_tensors(*_philox(c0, c1, rng[1] & M32, (rng[1] >> 32) & M32, rng)), -1)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1).view(rows, -1)[:, :cols]
    return halves < d, 65536.0 / (65536 - d)


def _act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain_linear(s):
    c = s["case"]
    T, n, k, dt = c["tokens"], c["n"], c["k"], DT[c["dtype"]]
    # the weights enter the product in the activations' type
    W = s["param"][:n * k].view(n, k).to(dt).float()
    if c["dir"] == "forward":
        z = s["x"].float() @ W.T + s["param"][-n:].float()
        y = _act(z, c["act"])
        if c["drop"] > 0:
            gone, factor = _dropped(T, n, c["drop"], s["rng"])
            y = torch.where(gone, 0.0, y * factor)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt), "pre": z.to(dt)} if c["pre"] else {"y": y.to(dt)}
    dz = s["dy"].float()
    if c["drop"] > 0:
        gone, factor = _dropped(T, n, c["drop"], s["rng"])
        dz = torch.where(gone, 0.0, dz * factor)
    if s["pre"] is not None:
        dz = dz * _act_slope(s["pre"].float(), c["act"])
    return {"dx": (dz @ W).to(dt), "dw": (dz.T @ s["x"].float()).to(dt), "db": dz.sum(0).to(dt)}


def _plain_dropout(s):
    c = s["case"]
    gone, factor = _dropped(c["rows"], c["cols"], c["drop"], s["rng"])
    y = torch.where(gone, 0.0, s["x"].float() * factor)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["x"].dtype)}


def _kept_below(case, n, m):
    """The threshold of a matrix: the compressor's own budget (rank 2) where keep is negative."""
    return (min((n + m) * 2, n * m) << 32) // (n * m) if case["keep"] < 0 else int(math.floor(case["keep"] * 2.0 ** 32 + 0.5))


def _plain_mask(s):
    c = s["case"]
    shapes = mask_shapes(c)
    off, N, L = placed(shapes)
    grad, err, out, rng = s["grad"], s["err"], s["out"], s["rng"]
    out[N:] = grad[:, N:N + L].float().mean(0).to(out.dtype)
    for t, shape in enumerate(shapes):
        if len(shape) == 1:
            continue
        n, m = shape
        at = slice(off[t], off[t] + n * m)
        c0 = torch.arange((n * m + 3) // 4, device=rng.device)
        words = torch.stack(torch.broadcast_tensors(*_philox(c0, torch.full_like(c0, t), rng[1] & M32, (rng[1] >> 32) & M32, rng)), -1)
        keep = words.view(-1)[:n * m] < _kept_below(c, n, m)
        M = grad[:, at].float() + err[:, at]
        delta = torch.where(keep, M.mean(0), 0.0)
        out[at] = delta.to(out.dtype)
        err[:, at] = M - delta
    return {"out": out, "err": err}


# ---- one call --------------------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"linear": _plain_linear, "dropout": _plain_dropout, "mask": _plain_mask}[c["op"]](s)
    from paper_1905_13727_amd import binding as B
    if c["op"] == "linear":
        plan, code = s["plan"], {"f32": B.PSGD_F32, "bf16": B.PSGD_BF16}
        shared = dict(bias=1, param_dtype=code[c["params"]], activation=c["act"], drop=c["drop"], rng=s["rng"], stream=s["stream"])
        if c["dir"] == "forward":
            plan.linear_forward(0, c["tokens"], s["param"], s["x"], s["y"], s["workspace"], residual=s["residual"], pre=s["pre"],
                                x_stride=s["x"].stride(0), residual_stride=c["n"] + c["pad"], **shared)
            return {"y": s["y"], "pre": s["pre"]} if c["pre"] else {"y": s["y"]}
        plan.linear_backward(0, c["tokens"], s["param"], s["x"], s["dy"], s["dx"], s["grad"], s["workspace"], pre=s["pre"],
                             x_stride=s["x"].stride(0), dy_stride=s["dy"].stride(0), **shared)
        n, k = c["n"], c["k"]
        return {"dx": s["dx"], "dw": s["grad"][:n * k].view(n, k), "db": s["grad"][_up(n * k, 64):][:n]}
    if c["op"] == "dropout":
        dtype = B.PSGD_BF16 if c["dtype"] == "bf16" else B.PSGD_F32
        if c["dir"] == "forward":
            B.dropout_forward(dtype, c["rows"], c["cols"], s["x"], s["y"], c["drop"], s["rng"], residual=s["residual"],
                              x_stride=s["x"].stride(0), residual_stride=c["cols"] + c["pad"], stream=s["stream"])
        else:
            B.dropout_backward(dtype, c["rows"], c["cols"], s["x"], s["y"], c["drop"], s["rng"], dy_stride=s["x"].stride(0),
                               stream=s["stream"])
        return {"y": s["y"]}
    s["plan"].random_mask_step(s["grad"], s["err"], c["keep"], s["rng"], s["out"], stream=s["stream"])
    return {"out": s["out"], "err": s["err"]}


def work(case):
    """Each input read once, each output written once.  The product: two operations per token, row and column, twice that
    in the backward pass.  Dropout and the mask: a multiplication and an addition per element."""
    z = SIZE[case["dtype"]]
    if case["op"] == "linear":
        T, n, k = case["tokens"], case["n"], case["k"]
        w = n * (k + 1) * SIZE[case["params"]]
        if case["dir"] == "forward":
            return {"bytes": w + z * T * (k + n * (1 + case["residual"] + case["pre"])), "flops": 2 * T * n * k}
        return {"bytes": w + z * (n * (k + 1) + T * (2 * k + n * (2 if case["act"] != "identity" else 1))), "flops": 4 * T * n * k}
    if case["op"] == "dropout":
        e = case["rows"] * case["cols"]
        return {"bytes": e * z * (2 + case["residual"]), "flops": 2 * e}
    _, N, L = placed(mask_shapes(case))
    W = case["workers"]
    return {"bytes": N * (W * (z + 8) + z) + L * (W + 1) * z, "flops": N * 3 * W}


# ---- the same in 64 bits, from the definition ------------------------------------------------------------------------

def _words64(c0, c1, seed, offset):
    """Philox4x32-10 with numpy's unsigned integers; c0 and c1 are uint64 arrays of one shape."""
    low, half = np.uint64(M32), np.uint64(32)
    c = [c0, c1, np.full_like(c0, offset & M32), np.full_like(c0, (offset >> 32) & M32)]
    for r in range(10):
        k0 = np.uint64(((seed & M32) + r * 0x9E3779B9) & M32)
        k1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & M32)
        hi0, lo0 = (c[0] * np.uint64(0xD2511F53)) >> half, (c[0] * np.uint64(0xD2511F53)) & low
        hi1, lo1 = (c[2] * np.uint64(0xCD9E8D57)) >> half, (c[2] * np.uint64(0xCD9E8D57)) & low
        c = [hi1 ^ c[1] ^ k0, lo1, hi0 ^ c[3] ^ k1, lo0]
    return np.stack(c, axis=-1)


def _keep_factor64(rows, cols, p, seed, offset, dev):
    """0 where an element is dropped, 1 / (1 - p) elsewhere, with p as the multiple of 2^-16 that it is rounded to."""
    d = int(math.floor(p * 65536 + 0.5))
    if d == 0:
        return 1.0
    groups = (cols + 7) // 8
    words = _words64(np.tile(np.arange(groups, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), groups), seed, offset)
    halves = np.ascontiguousarray(words.astype("<u4")).view("<u2").reshape(rows, groups * 8)[:, :cols]
    return torch.from_numpy(np.where(halves >= d, 65536.0 / (65536.0 - d), 0.0)).to(dev)


def exact(case, seed):
    s = prepare(case, seed)
    key, offset = int(s["rng"][0]), int(s["rng"][1])
    if case["op"] == "mask":
        shapes = mask_shapes(case)
        off, N, L = placed(shapes)
        if N > 32_000_000:
            return None
        g, e = s["grad"].double(), s["err"].double()
        out = torch.zeros(N + L, dtype=torch.float64, device=g.device)
        out[N:] = g[:, N:N + L].mean(0)
        for t, shape in enumerate(shapes):
            if len(shape) == 2:
                size = shape[0] * shape[1]
                counters = np.arange((size + 3) // 4, dtype=np.uint64)
                words = _words64(counters, np.full_like(counters, t), key, offset).reshape(-1)[:size]
                keep = torch.from_numpy(words < np.uint64(_kept_below(case, *shape))).to(g.device)
                at = slice(off[t], off[t] + size)
                e[:, at] += g[:, at]
                out[at] = e[:, at].mean(0) * keep
                e[:, at] -= out[at]
        return {"out": out, "err": e}
    if case["op"] == "dropout":
        y = s["x"].double() * _keep_factor64(case["rows"], case["cols"], case["drop"], key, offset, s["x"].device)
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    T, n, k = case["tokens"], case["n"], case["k"]
    W = s["param"][:n * k].to(DT[case["dtype"]]).double().reshape(n, k)
    x = s["x"].double()
    factor = _keep_factor64(T, n, case["drop"], key, offset, x.device)

    def curve(z):
        if case["act"] == "relu":
            return z.clamp(min=0)
        if case["act"] == "gelu":
            return z * 0.5 * torch.erfc(-z / math.sqrt(2))
        if case["act"] == "gelu_tanh":   # (1 + tanh u) / 2 is the logistic function of 2 u
            return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        if case["act"] == "silu":
            return z * torch.sigmoid(z)
        return z

    if case["dir"] == "forward":
        z = torch.addmm(s["param"][-n:].double(), x, W.T.contiguous())
        y = curve(z) * factor
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"y": y, "pre": z} if case["pre"] else {"y": y}
    dz = s["dy"].double() * factor
    if s["pre"] is not None:
        z = s["pre"].double()
        if case["act"] == "relu":
            dz = dz * (z > 0)
        else:
            z.requires_grad_(True)
            dz, = torch.autograd.grad(curve(z), z, dz)
    return {"dx": dz @ W, "dw": dz.T.contiguous() @ x, "db": dz.sum(0)}
