"""The layer operators of trained networks as measurable cases: affine layer with its epilogue, dropout, group norm.

A case is one call as a user of the library makes it next to a training run: evaluating the layers of a trained model on
data, or one layer's forward or backward pass in a network of the user's own.  Sizes are those of the configurations in
`inputs.config` (784-256-10, 4096 features, 60000 samples, 64 workers x 128 rows, 128 x 64 rows, 400-120-84-10, 32 x 32
images) or generic ones of the same kind.  Every operator also has a plain form in elementary torch operations (`own`
false), and `exact` gives its definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False


def _linear(M, n_in, n_out, dtype, act, **kw):
    c = dict(op="linear", M=M, n_in=n_in, n_out=n_out, dtype=dtype, act=act, residual=False, pre=False)
    c.update(kw)
    return c


def _linear_grad(M, n_in, n_out, dtype, act, **kw):
    return dict(op="linear_grad", M=M, n_in=n_in, n_out=n_out, dtype=dtype, act=act, **kw)


def _dropout(rows, cols, dtype, p, residual, **kw):
    return dict(op="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, **kw)


def _norm(N, H, W, C, groups, dtype, act, grad=False, **kw):
    return dict(op="group_norm_grad" if grad else "group_norm", N=N, H=H, W=W, C=C, groups=groups, dtype=dtype, act=act, **kw)


def listed():
    return [
        # configuration 3's hidden layer answering one sample: the smallest call, where latency counts
        _linear(1, 784, 256, "bf16", "relu", name="linear_one_row"),
        # its output layer over the whole dataset: ten classes, rows of results that are not 16-byte multiples
        _linear(60000, 256, 10, "bf16", "none", name="linear_classes"),
        # fp32, no size a multiple of anything, residual path and saved pre-activation of a training step
        _linear(1037, 785, 501, "fp32", "gelu", residual=True, pre=True, name="linear_ragged_fp32"),
        # a wide layer over the rows of 128 workers x 64, forward pass of a training step
        _linear(8192, 4096, 4096, "bf16", "silu", residual=True, pre=True, name="linear_wide"),
        # a small fp32 layer of odd widths (400-120-84-10 without its alignment), backward
        _linear_grad(1111, 401, 123, "fp32", "silu", name="linear_grad_ragged_fp32"),
        # the wide layer backward
        _linear_grad(8192, 4096, 4096, "bf16", "gelu", name="linear_grad_wide"),
        # one worker's minibatch of hidden activations
        _dropout(128, 256, "bf16", 0.5, False, name="dropout_minibatch"),
        # a whole dataset's activations, dropped and added to the residual path
        _dropout(60000, 1024, "bf16", 0.1, True, name="dropout_wide"),
        # feature maps behind the first convolution of the paper's model (28 x 28 x 6), odd channel groups, fp32
        _norm(20, 28, 28, 6, 3, "fp32", "relu", name="group_norm_conv1"),
        # large feature maps of a residual network
        _norm(64, 64, 64, 320, 32, "bf16", "silu", name="group_norm_wide"),
        # backward, fp32, odd sizes
        _norm(13, 31, 29, 84, 7, "fp32", "gelu", grad=True, name="group_norm_grad_ragged_fp32"),
        # backward over a batch of 32 x 32 maps
        _norm(128, 32, 32, 256, 32, "bf16", "silu", grad=True, name="group_norm_grad_wide"),
    ]


ACTS = ("none", "relu", "gelu", "silu")


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "linear_grad", "dropout", "group_norm", "group_norm_grad"])
    dtype = "bf16" if rng.random() < 0.65 else "fp32"
    odd = rng.random() < 0.35
    size = (lambda v: v) if odd else (lambda v: max(8, v // 8 * 8))
    act = rng.choice(ACTS)
    if op in ("linear", "linear_grad"):
        n_in, n_out = size(_log(rng, 16, 4096)), size(_log(rng, 2, 4096))
        limit = 1.3e11 if dtype == "bf16" else 2e10                 # multiply-adds of one product
        M = max(1, min(_log(rng, 1, 60000), int(limit / (n_in * n_out))))
        M = max(1, min(M, (5 if dtype == "bf16" else 2) * 10 ** 7 // (n_in + 2 * n_out)))
        if op == "linear":
            return _linear(M, n_in, n_out, dtype, act, residual=rng.random() < 0.5, pre=rng.random() < 0.5)
        return _linear_grad(M, n_in, n_out, dtype, act)
    if op == "dropout":
        cols = size(_log(rng, 2, 8192))
        rows = max(1, min(_log(rng, 1, 60000), (6 if dtype == "bf16" else 3) * 10 ** 7 // cols))
        return _dropout(rows, cols, dtype, round(rng.uniform(0.02, 0.7), 3), rng.random() < 0.5)
    groups = rng.choice([1, 2, 3, 7, 8, 16, 32])
    C = groups * (rng.choice([1, 2, 3, 5, 6, 12, 20]) if odd else rng.choice([2, 4, 8, 10, 16]))
    H, W = _log(rng, 4, 96), _log(rng, 4, 96)
    most = (8 if op == "group_norm" else 3) * 10 ** 7 // (1 if dtype == "bf16" else 2)
    N = max(1, min(_log(rng, 1, 128), most // (H * W * C)))
    return _norm(N, H, W, C, groups, dtype, act, grad=op == "group_norm_grad")


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    store = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(store)

    def empty(*shape, dtype=store):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    s = dict(case=case)
    if case["op"] in ("linear", "linear_grad"):
        M, n_in, n_out = case["M"], case["n_in"], case["n_out"]
        s["x"] = randn(M, n_in).clamp_(min=-0.5)                     # activations of the layer below
        s["w"] = randn(n_in, n_out, scale=math.sqrt(2.0 / n_in))     # He-normal
        s["b"] = randn(n_out, scale=0.1)
        if case["op"] == "linear":
            s["r"] = randn(M, n_out) if case["residual"] else None
            s["z"] = empty(M, n_out) if case["pre"] else None
            s["y"] = empty(M, n_out)
        else:
            s["dy"] = randn(M, n_out, scale=1.0 / M)
            s["z"] = (s["x"].float() @ s["w"].float() + s["b"].float()).to(store) if case["act"] != "none" else None
            s["dx"], s["dw"], s["db"] = empty(M, n_in), empty(n_in, n_out), empty(n_out)
    elif case["op"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = randn(rows, cols)
        s["r"] = randn(rows, cols) if case["residual"] else None
        s["y"] = empty(rows, cols)
        s["seed"], s["call"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), seed % 1000
    else:
        N, H, W, C, G = case["N"], case["H"], case["W"], case["C"], case["groups"]
        shift = torch.randn(C, generator=g, device="cuda")
        s["x"] = (torch.randn(N, H, W, C, generator=g, device="cuda") + shift).to(store)   # channels have means of their own
        s["w"], s["b"] = (1.0 + 0.1 * torch.randn(C, generator=g, device="cuda")).to(store), randn(C, scale=0.1)
        if case["op"] == "group_norm":
            s["y"] = empty(N, H, W, C)
            s["mean"], s["rstd"] = empty(N, G, dtype=torch.float32), empty(N, G, dtype=torch.float32)
        else:
            xs = s["x"].float().view(N, H * W, G, C // G)
            s["mean"] = xs.mean(dim=(1, 3)).contiguous()
            s["rstd"] = torch.rsqrt(xs.var(dim=(1, 3), unbiased=False) + EPS).contiguous()
            s["dy"] = randn(N, H, W, C, scale=1.0 / N)
            s["dx"], s["dw"], s["db"] = empty(N, H, W, C), empty(C), empty(C)
    return s


EPS = 1e-5
_M32 = 0xFFFFFFFF


def _keep_plain(rows, cols, p, seed, call):
    """Dropout's mask: 16 bits per element of the Philox4x32-10 block (column / 8, row, 2, call), key = seed."""
    nblk = (cols + 7) // 8
    c = [torch.arange(nblk, device="cuda", dtype=torch.int64)[None, :].expand(rows, nblk),
         torch.arange(rows, device="cuda", dtype=torch.int64)[:, None].expand(rows, nblk),
         torch.full((rows, nblk), 2, device="cuda", dtype=torch.int64),
         torch.full((rows, nblk), call, device="cuda", dtype=torch.int64)]
    k0, k1 = seed & _M32, seed >> 32
    for _ in range(10):                                              # (products modulo 2^64 have the right 64 bits)
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & _M32) ^ c[1] ^ k0, b & _M32, ((a >> 32) & _M32) ^ c[3] ^ k1, a & _M32]
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    half = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=-1).reshape(rows, nblk * 8)[:, :cols]
    return half >= _threshold(p)


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _run_plain(s):
    c = s["case"]
    store = s["x"].dtype
    x = s["x"].float()
    if c["op"] == "linear":
        z = x @ s["w"].float() + s["b"].float()
        y = _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return (y.to(store),) + ((z.to(store),) if c["pre"] else ())
    if c["op"] == "linear_grad":
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _act_slope(s["z"].float(), c["act"])
        return (dz @ s["w"].float().t()).to(store), (x.t() @ dz).to(store), dz.sum(dim=0).to(store)
    if c["op"] == "dropout":
        keep = _keep_plain(c["rows"], c["cols"], c["p"], s["seed"], s["call"])
        y = torch.where(keep, x * (65536.0 / (65536 - _threshold(c["p"]))), torch.zeros_like(x))
        if s["r"] is not None:
            y = y + s["r"].float()
        return y.to(store)
    N, C, G = c["N"], c["C"], c["groups"]
    x = x.view(N, -1, G, C // G)
    w, b = s["w"].float().view(G, C // G), s["b"].float().view(G, C // G)
    if c["op"] == "group_norm":
        n = x.shape[1] * x.shape[3]
        mean = x.sum(dim=(1, 3)) / n
        x = x - mean[:, None, :, None]
        rstd = 1.0 / torch.sqrt((x * x).sum(dim=(1, 3)) / n + EPS)
        y = _act(x * rstd[:, None, :, None] * w + b, c["act"])
        return y.reshape(s["x"].shape).to(store), mean, rstd
    rstd = s["rstd"][:, None, :, None]
    xh = (x - s["mean"][:, None, :, None]) * rstd
    g = s["dy"].float().view(x.shape)
    u = xh * w + b
    if c["act"] == "relu":                                           # (which side of zero: decided in 64 bits)
        x64, m64, r64 = x.double(), s["mean"].double()[:, None, :, None], rstd.double()
        u = (x64 - m64) * r64 * w.double() + b.double()
    if c["act"] != "none":
        g = g * _act_slope(u, c["act"]).float()
    dw, db = (g * xh).sum(dim=(0, 1)).reshape(C), g.sum(dim=(0, 1)).reshape(C)
    g = g * w
    n = x.shape[1] * x.shape[3]
    s1, s2 = g.sum(dim=(1, 3), keepdim=True) / n, (g * xh).sum(dim=(1, 3), keepdim=True) / n
    dx = rstd * (g - s1 - xh * s2)
    return dx.reshape(s["x"].shape).to(store), dw.to(store), db.to(store)


def run(state):
    if not own:
        return _run_plain(state)
    from paper_2301_08895_b200 import abs as gpu
    s, c = state, state["case"]
    op = c["op"]
    if op == "dropout":
        gpu.dropout(s["x"], s["r"], s["y"], c["p"], s["seed"], s["call"])
        return s["y"]
    act = {"none": gpu.ACT_NONE, "relu": gpu.ACT_RELU, "gelu": gpu.ACT_GELU, "silu": gpu.ACT_SILU}[c["act"]]
    if op == "linear":
        gpu.linear(s["x"], s["w"], s["b"], s["r"], s["y"], act, pre=s["z"])
        return (s["y"],) + ((s["z"],) if c["pre"] else ())
    if op == "linear_grad":
        gpu.linear_grad(s["dy"], s["x"], s["w"], s["z"], s["dx"], s["dw"], s["db"], act)
        return s["dx"], s["dw"], s["db"]
    if op == "group_norm":
        gpu.group_norm(s["x"], c["groups"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], EPS, act)
        return s["y"], s["mean"], s["rstd"]
    gpu.group_norm_grad(s["dy"], s["x"], c["groups"], s["w"], s["b"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], act)
    return s["dx"], s["dw"], s["db"]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("linear", "linear_grad"):
        M, n_in, n_out = case["M"], case["n_in"], case["n_out"]
        rows, weights = M * (n_in + n_out), n_in * n_out + n_out
        if case["op"] == "linear":
            return {"bytes": float(e * (rows + weights + M * n_out * (int(case["residual"]) + int(case["pre"])))),
                    "flops": 2.0 * M * n_in * n_out}
        return {"bytes": float(e * (rows + M * n_in + 2 * weights - n_out + M * n_out * int(case["act"] != "none"))),
                "flops": 4.0 * M * n_in * n_out}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": float(e * n * (2 + int(case["residual"]))), "flops": 2.0 * n}
    n, C, stats = case["N"] * case["H"] * case["W"] * case["C"], case["C"], 8 * case["N"] * case["groups"]
    if case["op"] == "group_norm":
        return {"bytes": float(e * (2 * n + 2 * C) + stats), "flops": 8.0 * n}
    return {"bytes": float(e * (3 * n + 4 * C) + stats), "flops": 16.0 * n}


# ---- the operators' definitions in 64 bits

def _phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _value64(z, act):
    return {"none": lambda: z, "relu": lambda: torch.clamp(z, min=0.0), "gelu": lambda: z * _phi(z),
            "silu": lambda: z * torch.special.expit(z)}[act]()


def _slope64(z, act):
    if act == "gelu":
        return _phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return torch.special.expit(z) + z * torch.special.expit(z) * torch.special.expit(-z)
    return torch.ones_like(z) if act == "none" else torch.where(z > 0, 1.0, 0.0).to(z.dtype)


def _keep64(rows, cols, p, seed, call):
    u, low = np.uint64, np.uint64(_M32)
    nblk = -(-cols // 8)
    c0, c1 = np.meshgrid(np.arange(nblk, dtype=u), np.arange(rows, dtype=u))
    c0, c1 = c0.ravel(), c1.ravel()
    c2, c3 = np.full_like(c0, 2), np.full_like(c0, call)
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        p0, p1 = c0 * u(3528531795), c2 * u(3449720151)
        c0, c1 = (p1 >> u(32)) ^ c1 ^ u(key[0]), p1 & low
        c2, c3 = (p0 >> u(32)) ^ c3 ^ u(key[1]), p0 & low
        key = [(key[0] + 2654435769) % 2 ** 32, (key[1] + 3144134277) % 2 ** 32]
    words = np.stack([c0, c1, c2, c3], axis=1).astype("<u4")
    return (words.view("<u2").reshape(rows, nblk * 8)[:, :cols]).astype(np.int64) >= round(65536 * p)


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    act = case.get("act")
    if case["op"] == "linear":
        z = torch.addmm(d["b"], d["x"], d["w"])
        y = _value64(z, act) + (d["r"] if case["residual"] else 0.0)
        return (y, z) if case["pre"] else (y,)
    if case["op"] == "linear_grad":
        dz = d["dy"] * _slope64(d["z"], act) if act != "none" else d["dy"]
        return torch.mm(dz, d["w"].T), torch.mm(d["x"].T, dz), dz.sum(0)
    if case["op"] == "dropout":
        keep = torch.from_numpy(_keep64(case["rows"], case["cols"], case["p"], s["seed"], s["call"])).cuda()
        kept = 1.0 - round(65536 * case["p"]) / 65536.0
        return keep * d["x"] / kept + (d["r"] if case["residual"] else 0.0)
    N, C, G = case["N"], case["C"], case["groups"]
    per_group = lambda t: t.reshape(N, -1, G, C // G).permute(0, 2, 1, 3).reshape(N, G, -1)      # noqa: E731
    back = lambda t: t.reshape(N, G, -1, C // G).permute(0, 2, 1, 3).reshape(N, -1, C)           # noqa: E731
    x = per_group(d["x"])
    if case["op"] == "group_norm":
        mean, var = x.mean(-1), x.var(-1, correction=0)
        xh = back((x - mean[..., None]) / torch.sqrt(var[..., None] + EPS))
        return _value64(xh * d["w"] + d["b"], act).reshape(d["x"].shape), mean, (var + EPS) ** -0.5
    xh = (x - d["mean"][..., None]) * d["rstd"][..., None]
    u = back(xh) * d["w"] + d["b"]
    g = d["dy"].reshape(N, -1, C) * _slope64(u, act)
    gw = per_group(g * d["w"])
    dx = d["rstd"][..., None] * (gw - gw.mean(-1, keepdim=True) - xh * (gw * xh).mean(-1, keepdim=True))
    return back(dx).reshape(d["x"].shape), (g * back(xh)).sum((0, 1)), g.sum((0, 1))
