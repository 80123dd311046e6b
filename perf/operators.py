"""Performance cases of the operators of a transformer's feed-forward part:
layer norm, the gated feed-forward block, and low-rank adapters beside a
shared projection.

With `own` false, `run` computes a case from elementary torch operations in 32
bits, rounded once at the end; with `own` true it calls the tensor entry
points of paper_2608_10803_amd, into output buffers that a program keeps.

A case is one of five kinds:
  norm        Y = (X - mean) rstd w + b over the rows of X, with the rows'
              mean and rstd
  norm_train  the same and its backward pass: dX, dw, db
  ffn         H = act(X Wg) * (X Wu), Y = H Wd
  ffn_train   the same and its backward pass: dX, dWg, dWu, dWd
  adapter     Y = X W + scale[a] (X down[a]^T) up[a]^T, a = index[row]; a row
              of index -1 has no adapter
Weights are D x F (F x D) matrices, "r": contiguous rows, "c": transposed
views, as a linear layer stores its weights.
"""
import math

import torch

own = False

# no drawn case does more than the largest listed ones
MAX_FLOPS = 4.4e12
MAX_BYTES = 3.6e9
MAX_NORM_BYTES = 1.0e9


def _norm(name, rows, cols, dtype="bf16", wtype="32", train=False):
    return {"name": name, "kind": "norm_train" if train else "norm", "rows": rows, "cols": cols, "dtype": dtype,
            "wtype": wtype}


def _ffn(name, M, D, F, dtype="bf16", layout="c", act="silu", train=False):
    return {"name": name, "kind": "ffn_train" if train else "ffn", "M": M, "D": D, "F": F, "dtype": dtype,
            "layout": layout, "act": act}


def _adapter(name, M, N, K, n, R, requests, dtype="bf16", layout="c"):
    return {"name": name, "kind": "adapter", "M": M, "N": N, "K": K, "n": n, "R": R, "requests": requests,
            "dtype": dtype, "layout": layout}


def listed():
    return [
        # decode: the norm before a block, 16 sequences
        _norm("norm_decode", 16, 4096),
        # odd rows and columns, 16-bit weights
        _norm("norm_odd", 4099, 1531, dtype="f16", wtype="16"),
        # training: 8192 tokens of a 4096-wide model
        _norm("norm_train", 8192, 4096, train=True),
        # decode of a small expert's block, one token
        _ffn("ffn_token_small", 1, 512, 1536),
        # decode: a batch of 16 sequences
        _ffn("ffn_decode", 16, 4096, 14336),
        # prefill: a chunk of 2048 tokens
        _ffn("ffn_prefill", 2048, 4096, 14336),
        # training an odd-sized block on a ragged number of tokens
        _ffn("ffn_train_odd", 1777, 1001, 2731, dtype="f16", layout="r", act="gelu", train=True),
        # training: 4096 tokens
        _ffn("ffn_train", 4096, 4096, 14336, train=True),
        # decode: one token of each of 16 requests, each with one of 16 adapters
        _adapter("adapter_decode", 16, 4096, 4096, 16, 16, 16),
        # decode: 64 requests over 32 adapters of rank 64, up-projection
        _adapter("adapter_decode_wide", 64, 14336, 4096, 32, 64, 64),
        # prompts of 6 requests and the single tokens of 30 others in one batch, odd rank
        _adapter("adapter_mixed", 1100, 4096, 4096, 24, 20, 36, dtype="f16", layout="r"),
        # prefill: 4096 tokens of 8 requests
        _adapter("adapter_prefill", 4096, 14336, 4096, 8, 16, 8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice(["norm", "norm_train", "ffn", "ffn", "ffn_train", "ffn_train", "adapter", "adapter", "adapter"])
    grain = rng.choice([1, 8, 64, 64])  # odd sizes and those of laid-out layers

    def dim(lo, hi):
        return max(lo, _log(rng, lo, hi) // grain * grain)

    dtype = rng.choice(["bf16", "bf16", "f16"])
    layout = rng.choice(["r", "c", "c"])
    if kind.startswith("norm"):
        c = _norm("", _log(rng, 1, 16384), dim(64, 16384), rng.choice([dtype, dtype, "f32"]), rng.choice(["16", "32"]),
                  kind == "norm_train")
        if c["dtype"] == "f32":
            c["wtype"] = "32"
    elif kind == "ffn":
        c = _ffn("", _log(rng, 1, 4096), dim(256, 8192), dim(256, 16384), dtype, layout,
                 rng.choice(["silu", "gelu", "gelu_tanh"]))
    elif kind == "ffn_train":
        c = _ffn("", _log(rng, 64, 8192), dim(256, 4096), dim(256, 14336), dtype, layout,
                 rng.choice(["silu", "gelu", "gelu_tanh"]), True)
    else:
        M = _log(rng, 1, 4096)
        c = _adapter("", M, dim(256, 14336), dim(256, 8192), _log(rng, 1, 64), _log(rng, 4, 64), min(M, _log(rng, 1, 64)),
                     dtype, layout)
    c.pop("name")
    return c


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        if (w["flops"] <= MAX_FLOPS and w["bytes"] <= (MAX_NORM_BYTES if c["kind"].startswith("norm") else MAX_BYTES)
                and 3072 not in c.values()):
            return c


_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _values(g, rows, cols, scale, dt):
    return torch.empty(rows, cols, device="cuda", dtype=torch.float32).normal_(0.0, scale, generator=g).to(dt)


def _weight(g, rows, cols, scale, dt, layout):
    """rows x cols; "c": a transposed view of a cols x rows tensor."""
    return _values(g, cols, rows, scale, dt).t() if layout == "c" else _values(g, rows, cols, scale, dt)


def _like(w):
    """An output buffer of the type and layout of the weight w."""
    if w.stride(0) == 1 and w.shape[0] > 1:
        return torch.empty(w.shape[1], w.shape[0], device="cuda", dtype=w.dtype).t()
    return torch.empty(w.shape, device="cuda", dtype=w.dtype)


def prepare(case, seed):
    """Activations of about unit variance (for the norms with an offset and a
    scale of their own in every row), weights of variance 1 / fan-in, and the
    output buffers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    s = {"kind": case["kind"], "dt": dt}
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        wt = dt if case["wtype"] == "16" else torch.float32
        x = _values(g, rows, cols, 1.0, torch.float32)
        x.mul_(_values(g, rows, 1, 0.3, torch.float32).exp_()).add_(_values(g, rows, 1, 0.5, torch.float32))
        s["X"] = x.to(dt)
        s["w"] = (_values(g, 1, cols, 0.2, torch.float32) + 1.0).view(cols).to(wt)
        s["b"] = _values(g, 1, cols, 0.2, wt).view(cols)
        s["eps"] = 1e-5
        s["Y"] = torch.empty(rows, cols, device="cuda", dtype=dt)
        s["mean"] = torch.empty(rows, device="cuda", dtype=torch.float32)
        s["rstd"] = torch.empty(rows, device="cuda", dtype=torch.float32)
        if case["kind"] == "norm_train":
            s["dY"] = _values(g, rows, cols, rows ** -0.5, dt)
            s["dX"] = torch.empty(rows, cols, device="cuda", dtype=dt)
            s["dw"] = torch.empty(cols, device="cuda", dtype=wt)
            s["db"] = torch.empty(cols, device="cuda", dtype=wt)
    elif case["kind"].startswith("ffn"):
        M, D, F = case["M"], case["D"], case["F"]
        s["act"] = case["act"]
        s["X"] = _values(g, M, D, 1.0, dt)
        s["Wg"] = _weight(g, D, F, D ** -0.5, dt, case["layout"])
        s["Wu"] = _weight(g, D, F, D ** -0.5, dt, case["layout"])
        s["Wd"] = _weight(g, F, D, F ** -0.5, dt, case["layout"])
        s["H"] = torch.empty(M, F, device="cuda", dtype=dt)
        s["Y"] = torch.empty(M, D, device="cuda", dtype=dt)
        if case["kind"] == "ffn_train":
            s["dY"] = _values(g, M, D, M ** -0.5, dt)
            s["gate"] = torch.empty(M, F, device="cuda", dtype=dt)
            s["up"] = torch.empty(M, F, device="cuda", dtype=dt)
            s["dX"] = torch.empty(M, D, device="cuda", dtype=dt)
            for n in ("Wg", "Wu", "Wd"):
                s["d" + n] = _like(s[n])
    else:
        M, N, K, n, R = case["M"], case["N"], case["K"], case["n"], case["R"]
        s["X"] = _values(g, M, K, 1.0, dt)
        s["W"] = _weight(g, K, N, K ** -0.5, dt, case["layout"])
        s["down"] = _values(g, n * R, K, K ** -0.5, dt).view(n, R, K)
        s["up"] = _values(g, n * N, R, 0.5 * R ** -0.5, dt).view(n, N, R)
        s["scale"] = _values(g, 1, n, 0.2, torch.float32).view(n).exp_()
        s["index"] = _rows_of_requests(case, seed).cuda()
        s["Y"] = torch.empty(M, N, device="cuda", dtype=dt)
    return s


def _rows_of_requests(case, seed):
    """The adapter of every row: each request owns a run of rows and one
    adapter (one request in eight has none). Where there are more rows than
    requests, one request in six is a prompt and the prompts share the rows
    that the others' single tokens leave."""
    r = torch.Generator().manual_seed(seed)
    M, req = case["M"], min(case["requests"], case["M"])
    lengths = torch.ones(req, dtype=torch.int64)
    prompts = req if M >= 64 * req else max(1, req // 6)
    share = torch.rand(prompts, generator=r) + 0.1
    extra = (share / share.sum() * (M - req)).floor().long()
    extra[0] += M - req - int(extra.sum())
    lengths[torch.randperm(req, generator=r)[:prompts]] += extra
    which = torch.randint(0, case["n"], (req,), generator=r)
    which[torch.rand(req, generator=r) < 0.125] = -1
    return torch.repeat_interleave(which, lengths).to(torch.int32)


def _act(name, x):
    """The activation and its derivative."""
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-x))
        return x * p, p * (1.0 + x * (1.0 - p))
    if name == "gelu":
        p = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
        return x * p, p + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    c, a = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(c * (x + a * x * x * x))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3.0 * a * x * x)


def _run_plain(s):
    dt = s["dt"]
    if s["kind"].startswith("norm"):
        x, w, b = s["X"].float(), s["w"].float(), s["b"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = ((d * d).mean(1, keepdim=True) + s["eps"]).rsqrt()
        xh = d * rstd
        y = (xh * w + b).to(dt)
        if s["kind"] == "norm":
            return y, mean.view(-1), rstd.view(-1)
        dy = s["dY"].float()
        wdy = dy * w
        dx = (wdy - wdy.mean(1, keepdim=True) - xh * (wdy * xh).mean(1, keepdim=True)) * rstd
        return y, dx.to(dt), (dy * xh).sum(0).to(s["w"].dtype), dy.sum(0).to(s["w"].dtype)
    if s["kind"].startswith("ffn"):
        x, wg, wu, wd = s["X"].float(), s["Wg"].float(), s["Wu"].float(), s["Wd"].float()
        gate, up = x @ wg, x @ wu
        a, da = _act(s["act"], gate)
        h = a * up
        y = (h @ wd).to(dt)
        if s["kind"] == "ffn":
            return y, h.to(dt)
        dy = s["dY"].float()
        dh = dy @ wd.t()
        dg, du = dh * up * da, dh * a
        dx = (dg @ wg.t() + du @ wu.t()).to(dt)
        return y, dx, (x.t() @ dg).to(dt), (x.t() @ du).to(dt), (h.t() @ dy).to(dt)
    x, n, R = s["X"].float(), s["down"].shape[0], s["down"].shape[1]
    y = x @ s["W"].float()
    # every row against every adapter, all but its own then dropped
    t = (x @ s["down"].float().view(n * R, -1).t()).view(-1, n, R)
    mine = (s["index"][:, None] == torch.arange(n, device="cuda", dtype=torch.int32)[None, :]).float()
    t = t * (mine * s["scale"][None, :])[:, :, None]
    up = s["up"].float().permute(0, 2, 1).reshape(n * R, -1)
    return (y + t.view(-1, n * R) @ up).to(dt)


def _run_own(s):
    import paper_2608_10803_amd as ac
    if s["kind"].startswith("norm"):
        ac.layer_norm_tensors(s["X"], s["w"], s["b"], s["Y"], eps=s["eps"], mean=s["mean"], rstd=s["rstd"])
        if s["kind"] == "norm":
            return s["Y"], s["mean"], s["rstd"]
        ac.layer_norm_backward_tensors(s["dY"], s["X"], s["w"], s["mean"], s["rstd"], s["dX"], dweight=s["dw"],
                                       dbias=s["db"])
        return s["Y"], s["dX"], s["dw"], s["db"]
    if s["kind"] == "ffn":
        return ac.gated_ffn_tensors(s["X"], s["Wg"], s["Wu"], s["Wd"], s["H"], s["Y"], act=s["act"]), s["H"]
    if s["kind"] == "ffn_train":
        ac.gated_ffn_tensors(s["X"], s["Wg"], s["Wu"], s["Wd"], s["H"], s["Y"], act=s["act"], gate=s["gate"],
                             up=s["up"])
        ac.gated_ffn_backward_tensors(s["dY"], s["X"], s["Wg"], s["Wu"], s["Wd"], s["gate"], s["up"], s["H"],
                                      dX=s["dX"], dWg=s["dWg"], dWu=s["dWu"], dWd=s["dWd"], act=s["act"])
        return s["Y"], s["dX"], s["dWg"], s["dWu"], s["dWd"]
    return ac.adapter_mm_tensors(s["X"], s["W"], s["down"], s["up"], s["index"], s["Y"], scale=s["scale"])


def run(s):
    return _run_own(s) if own else _run_plain(s)


def work(case):
    if case["kind"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        e = 4 if case["dtype"] == "f32" else 2
        w = e if case["wtype"] == "16" else 4
        if case["kind"] == "norm":
            return {"bytes": 2 * e * rows * cols + 2 * w * cols + 8 * rows, "flops": 8 * rows * cols}
        return {"bytes": 4 * e * rows * cols + 4 * w * cols, "flops": 22 * rows * cols}
    if case["kind"] == "ffn":
        M, D, F = case["M"], case["D"], case["F"]
        return {"bytes": 2 * (2 * M * D + M * F + 3 * D * F), "flops": 6 * M * D * F}
    if case["kind"] == "ffn_train":
        M, D, F = case["M"], case["D"], case["F"]
        # in: X, dY, weights; out: Y, dX, the gradients
        return {"bytes": 2 * (4 * M * D + 6 * D * F), "flops": 18 * M * D * F}
    M, N, K, n, R = case["M"], case["N"], case["K"], case["n"], case["R"]
    used = min(n, case["requests"])
    return {"bytes": 2 * (M * K + K * N + M * N + used * R * (K + N)), "flops": 2 * M * (N * K + R * (K + N))}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)

    def f64(n):
        return s[n].to(torch.float64)

    if case["kind"].startswith("norm"):
        x, w = f64("X"), f64("w")
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + s["eps"])
        xh = (x - mean[:, None]) * rstd[:, None]
        y = xh * w + f64("b")
        if case["kind"] == "norm":
            return y, mean, rstd
        dy = f64("dY")
        # the gradient of x_hat through the projections off 1 and x_hat
        p = dy * w
        c = p.shape[1]
        dx = rstd[:, None] * (p - p.sum(1)[:, None] / c - xh * ((p * xh).sum(1)[:, None] / c))
        return y, dx, torch.sum(dy * xh, 0), torch.sum(dy, 0)
    if case["kind"].startswith("ffn"):
        x, wg, wu, wd = f64("X"), f64("Wg"), f64("Wu"), f64("Wd")
        z = (x @ wg).requires_grad_(case["kind"] == "ffn_train")
        if case["act"] == "silu":
            a = z * torch.sigmoid(z)
        elif case["act"] == "gelu":
            a = z * (1.0 - torch.erfc(z / math.sqrt(2.0)) / 2.0)
        else:
            a = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
        u = x @ wu
        h = a.detach() * u
        y = h @ wd
        if case["kind"] == "ffn":
            return y, h
        dy = f64("dY")
        dh = dy @ wd.t()
        dwd = h.t() @ dy
        du = dh * a.detach()
        dz, = torch.autograd.grad(a, z, dh * u)
        del h, dh, u, a, z
        dx = dz @ wg.t()
        dx += du @ wu.t()
        return y, dx, x.t() @ dz, x.t() @ du, dwd
    x = f64("X")
    y = x @ f64("W")
    for a in range(case["n"]):
        rows = (s["index"] == a).nonzero().view(-1)
        if rows.numel():
            t = x[rows] @ s["down"][a].to(torch.float64).t()
            y[rows] += s["scale"][a].to(torch.float64) * (t @ s["up"][a].to(torch.float64).t())
    return y
