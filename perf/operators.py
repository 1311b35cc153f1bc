"""Operators of language models that training steps and answers need beside products and recurrent layers, as cases
that can be timed and compared.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass: in plain torch
where `own` is false, by the framework's entry points where it is true.  `work` counts the bytes and operations that the
pass cannot do without, `exact` has the same results from the definition in 64 bits.

Operators (x, y, ... are matrices whose rows are one token, or one example, each):
  layer_norm     y = (x - mean) * rstd * gamma + beta over every row, with mean and rstd; backward dx, dgamma, dbeta
  dropout        y = (residual +) keep * x / (1 - ratio), the mask drawn from a counter-based generator and never stored;
                 its backward is the same call on the gradient
  residual_norm  s = residual + dropout(x), y = layer_norm(s as it is stored) in one pass; backward from dy and the gradient
                 of s to dresidual, dx, dgamma, dbeta
  sample         one token a row from logits: temperature, top-k, top-p and min-p of the row, a given number in [0, 1)

The mask: element (row, col) of call site t is kept where word col % 4 of Philox-4x32 with seven rounds (Salmon et al., "Parallel
random numbers: as easy as 1, 2, 3"), key = the 64-bit seed, counter = (col / 4, row, offset, t), is at least
round(ratio * 2^32).
"""
import math

import numpy as np
import torch

own = False

F32, BF16, F64, I64 = torch.float32, torch.bfloat16, torch.float64, torch.int64
DT = {"f32": F32, "bf16": BF16}
M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
MASK = 0xFFFFFFFF
ROUNDS = 7
EPS = 1e-5


def listed():
    return [
        # One time step's hidden states of the recurrent language model (batch 128, 650 units): the smallest call.
        {"name": "norm_fwd_f32_128x650", "op": "layer_norm", "rows": 128, "cols": 650, "dtype": "f32", "out": "f32", "pad": 0, "backward": False},
        # All 35 steps' hidden states, forward and backward with the gradients of the weights.
        {"name": "norm_f32_4480x650", "op": "layer_norm", "rows": 4480, "cols": 650, "dtype": "f32", "out": "f32", "pad": 0, "backward": True},
        # A hidden layer of the wide MLP in mixed precision.
        {"name": "norm_bf16_8192x4096", "op": "layer_norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "out": "bf16", "pad": 0, "backward": True},
        # Few long rows of an odd length inside a wider buffer, normalised into bfloat16 from fp32.
        {"name": "norm_mixed_99x20011", "op": "layer_norm", "rows": 99, "cols": 20011, "dtype": "f32", "out": "bf16", "pad": 5, "backward": True},
        # Dropout of the language model's embeddings and their gradient.
        {"name": "dropout_f32_4480x650", "op": "dropout", "rows": 4480, "cols": 650, "dtype": "f32", "residual": False, "ratio": 0.5, "pad": 0},
        # A wide activation, added to the residual stream.
        {"name": "dropout_bf16_8192x4096", "op": "dropout", "rows": 8192, "cols": 4096, "dtype": "bf16", "residual": True, "ratio": 0.1, "pad": 0},
        # A residual block of the MNIST classifier's width.
        {"name": "residual_f32_1024x1000", "op": "residual_norm", "rows": 1024, "cols": 1000, "dtype": "f32", "stream": "f32", "ratio": 0.1, "pad": 0},
        # A residual block of the wide MLP: activations in bfloat16, the stream in fp32.
        {"name": "residual_mixed_4096x4096", "op": "residual_norm", "rows": 4096, "cols": 4096, "dtype": "bf16", "stream": "f32", "ratio": 0.1, "pad": 0},
        # The same with all of it in bfloat16, the largest pass over rows.
        {"name": "residual_bf16_8192x4096", "op": "residual_norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "stream": "bf16", "ratio": 0.1, "pad": 0},
        # The language model answers: one token for each of its 128 sequences, vocabulary 10000.
        {"name": "sample_f32_128x10000", "op": "sample", "rows": 128, "vocab": 10000, "dtype": "f32", "spread": 2.5, "banned": 0.0,
         "temperature": True, "top_k": True, "top_p": False, "min_p": False, "pad": 0},
        # A single request with a large vocabulary, where latency counts.
        {"name": "sample_bf16_1x131072", "op": "sample", "rows": 1, "vocab": 131072, "dtype": "bf16", "spread": 2.5, "banned": 0.0,
         "temperature": True, "top_k": False, "top_p": True, "min_p": False, "pad": 0},
        # A full batch whose requests bring parameters of their own, some tokens banned.
        {"name": "sample_f32_256x131072", "op": "sample", "rows": 256, "vocab": 131072, "dtype": "f32", "spread": 2.5, "banned": 0.02,
         "temperature": True, "top_k": True, "top_p": True, "min_p": True, "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over the logarithm of its range: a third as drawn, a third multiples of 8, a third of 64."""
    n, step = _log(rng, lo, hi), rng.choice((1, 8, 64))
    return max(lo, min(hi, (n + step - 1) // step * step))


def draw(rng):
    op = rng.choice(("layer_norm", "layer_norm", "dropout", "residual_norm", "residual_norm", "sample", "sample"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "sample":
        vocab = _size(rng, 2, 131072)
        return {"op": op, "rows": _log(rng, 1, 256), "vocab": vocab, "dtype": dtype, "spread": round(rng.uniform(0.5, 5.0), 3),
                "banned": rng.choice((0.0, 0.02, 0.9)), "temperature": rng.random() < 0.8, "top_k": rng.random() < 0.5,
                "top_p": rng.random() < 0.5, "min_p": rng.random() < 0.3, "pad": rng.choice((0, 0, 1, 8))}
    cols = _size(rng, 16, 20480)
    rows = min(_size(rng, 1, 16384), max(1, 2 ** 24 // cols))
    pad = rng.choice((0, 0, 3, 8))
    case = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "pad": pad}
    if op == "layer_norm":
        case.update(out=rng.choice((dtype, "f32", "bf16")), backward=rng.random() < 0.7)
    else:
        case["ratio"] = rng.choice((0.0, 0.1, 0.25, 0.5, 0.9))
        if op == "dropout":
            case["residual"] = rng.random() < 0.5
        else:
            case["stream"] = rng.choice((dtype, "f32"))
    return case


# ---- what a program holds before the call -----------------------------------------------------------------------
def _rows(gen, case, dtype, scale=1.0, shift=0.0):
    """A matrix of values as layers leave them, inside a buffer whose rows are `pad` elements longer."""
    r, c, pad = case["rows"], case["cols"], case["pad"]
    buf = torch.randn(r, c + pad, generator=gen, device="cuda", dtype=F32)
    return (buf * scale + shift).to(DT[dtype])[:, :c]


def _like(x, dtype):
    """Memory for a result shaped and pitched like x."""
    return torch.empty(x.shape[0], x.stride(0), device="cuda", dtype=DT[dtype])[:, :x.shape[1]] if x.shape[0] > 1 else torch.empty(
        x.shape, device="cuda", dtype=DT[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    op = case["op"]
    if op == "sample":
        n, v = case["rows"], case["vocab"]
        z = torch.randn(n, v + case["pad"], generator=gen, device="cuda") * case["spread"]
        uniform = lambda: torch.rand(n, generator=gen, device="cuda")
        # a few tokens of each row stand out, as they do after training
        best = torch.randint(0, v, (n, 8), generator=gen, device="cuda")
        z.scatter_add_(1, best, torch.rand(n, 8, generator=gen, device="cuda") * 3 * case["spread"])
        if case["banned"] > 0:
            z.masked_fill_(torch.rand(z.shape, generator=gen, device="cuda") < case["banned"], -math.inf)
        st["logits"], st["u"] = z.to(DT[case["dtype"]])[:, :v], uniform()
        # parameters by row, some of them off: temperature 0 takes the best token, top_k 0 and top_p 1 and min_p 0 keep all
        off = lambda share: uniform() < share
        st["temperature"] = torch.where(off(0.1), torch.zeros(n, device="cuda"), 0.5 + uniform()) if case["temperature"] else None
        st["top_k"] = torch.where(off(0.2), torch.zeros(n, device="cuda"), 1 + 99 * uniform()).to(torch.int32) if case["top_k"] else None
        st["top_p"] = torch.where(off(0.2), torch.ones(n, device="cuda"), 0.5 + 0.49 * uniform()) if case["top_p"] else None
        st["min_p"] = torch.where(off(0.2), torch.zeros(n, device="cuda"), 0.02 + 0.1 * uniform()) if case["min_p"] else None
        if own:
            from paper_1908_00213_amd import binding as B
            st["out"] = torch.empty(n, device="cuda", dtype=I64)
            st["ws"] = torch.empty(max(256, B.sample_workspace_bytes(st["logits"])), device="cuda", dtype=torch.uint8)
        return st
    c = case["cols"]
    st["rng"] = torch.stack([torch.randint(0, 2 ** 62, (), generator=gen, device="cuda"), torch.randint(0, 2 ** 31, (), generator=gen, device="cuda")])
    st["site"] = 1 + seed % 7
    st["x"] = _rows(gen, case, case["dtype"], 1.5, 0.75)
    if op == "dropout":
        st["dy"] = _rows(gen, case, case["dtype"], 1e-3)
        st["residual"] = _rows(gen, case, case["dtype"]) if case["residual"] else None
        if own:
            st["y"], st["dx"] = _like(st["x"], case["dtype"]), _like(st["x"], case["dtype"])
        return st
    st["gamma"] = 1.0 + 0.1 * torch.randn(c, generator=gen, device="cuda")
    st["beta"] = 0.1 * torch.randn(c, generator=gen, device="cuda")
    plain = op == "layer_norm"
    st["dy"] = _rows(gen, case, case["out"] if plain else case["dtype"], 1e-2)
    if not plain:
        st["residual"], st["ds"] = _rows(gen, case, case["stream"], 1.0, 0.5), _rows(gen, case, case["stream"], 1e-2)
    if own:
        from paper_1908_00213_amd import binding as B
        n = case["rows"]
        st["mean"], st["rstd"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        st["y"], st["dx"] = _like(st["x"], case["out"] if plain else case["dtype"]), _like(st["x"], case["dtype"])
        st["dgamma"], st["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        if not plain:
            st["s"], st["dresidual"] = _like(st["x"], case["stream"]), _like(st["x"], case["stream"])
        st["ws"] = torch.empty(max(256, B.layer_norm_bwd_workspace_bytes(st["x"] if plain else st["s"])), device="cuda", dtype=torch.uint8)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _PLAIN[st["case"]["op"]](st)


def _run_own(st):
    from paper_1908_00213_amd import binding as B
    case = st["case"]
    op = case["op"]
    if op == "sample":
        return B.sample(st["logits"], st["u"], st["out"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                        min_p=st["min_p"], ws=st["ws"])
    if op == "dropout":
        B.dropout(st["x"], st["y"], case["ratio"], st["rng"], st["site"], residual=st["residual"])
        B.dropout(st["dy"], st["dx"], case["ratio"], st["rng"], st["site"])
        return st["y"], st["dx"]
    if op == "layer_norm":
        B.layer_norm_fwd(st["x"], st["y"], st["gamma"], st["beta"], EPS, st["mean"], st["rstd"])
        if not case["backward"]:
            return st["y"], st["mean"], st["rstd"]
        B.layer_norm_bwd(st["dy"], st["x"], st["mean"], st["rstd"], st["dx"], st["gamma"], st["dgamma"], st["dbeta"], ws=st["ws"])
        return st["y"], st["mean"], st["rstd"], st["dx"], st["dgamma"], st["dbeta"]
    B.residual_norm_fwd(st["x"], st["residual"], st["s"], st["y"], st["gamma"], st["beta"], EPS, st["mean"], st["rstd"],
                        ratio=case["ratio"], rng=st["rng"], site=st["site"])
    B.residual_norm_bwd(st["dy"], st["ds"], st["s"], st["mean"], st["rstd"], st["dresidual"], st["dx"], st["gamma"], st["dgamma"], st["dbeta"],
                        ratio=case["ratio"], rng=st["rng"], site=st["site"], ws=st["ws"])
    return st["s"], st["y"], st["mean"], st["rstd"], st["dresidual"], st["dx"], st["dgamma"], st["dbeta"]


def _mulhilo(m, a):
    """High and low half of the 64-bit product of two 32-bit numbers, held in 64-bit signed ones."""
    return (m * (a >> 16) + ((m * (a & 0xFFFF)) >> 16)) >> 16, (m * a) & MASK


def _kept(st):
    """The mask of (rows, cols) in torch's integers."""
    case = st["case"]
    n, c = case["rows"], case["cols"]
    seed, offset = st["rng"][0], st["rng"][1] & MASK
    k0, k1 = seed & MASK, (seed >> 32) & MASK
    c0 = torch.arange((c + 3) // 4, device="cuda")[None, :].expand(n, -1)
    c1 = torch.arange(n, device="cuda")[:, None].expand_as(c0)
    c2, c3 = offset.expand_as(c0), torch.full_like(offset, st["site"]).expand_as(c0)
    for _ in range(ROUNDS):
        (h0, l0), (h1, l1) = _mulhilo(M0, c0), _mulhilo(M1, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + W0) & MASK, (k1 + W1) & MASK
    words = torch.stack([c0, c1, c2, c3], -1).reshape(n, -1)[:, :c]
    return words >= int(math.floor(case["ratio"] * 2.0 ** 32 + 0.5))


def _plain_drop(st, x, kept):
    return torch.where(kept, x.float() * (1.0 / (1.0 - st["case"]["ratio"])), torch.zeros((), device="cuda"))


def _plain_dropout(st):
    dt = DT[st["case"]["dtype"]]
    kept = _kept(st)
    y = _plain_drop(st, st["x"], kept)
    if st["residual"] is not None:
        y = st["residual"].float() + y
    return y.to(dt), _plain_drop(st, st["dy"], kept).to(dt)


def _plain_norm(x, gamma, beta):
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + EPS)
    return d * rstd[:, None] * gamma + beta, mean, rstd


def _plain_norm_bwd(dy, x, mean, rstd, gamma):
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def _plain_layer_norm(st):
    case = st["case"]
    x = st["x"].float()
    y, mean, rstd = _plain_norm(x, st["gamma"], st["beta"])
    y = y.to(DT[case["out"]])
    if not case["backward"]:
        return y, mean, rstd
    dx, dgamma, dbeta = _plain_norm_bwd(st["dy"].float(), x, mean, rstd, st["gamma"])
    return y, mean, rstd, dx.to(DT[case["dtype"]]), dgamma, dbeta


def _plain_residual_norm(st):
    case = st["case"]
    layer, stream = DT[case["dtype"]], DT[case["stream"]]
    kept = _kept(st)
    s = (st["residual"].float() + _plain_drop(st, st["x"], kept)).to(stream)
    y, mean, rstd = _plain_norm(s.float(), st["gamma"], st["beta"])
    ds, dgamma, dbeta = _plain_norm_bwd(st["dy"].float(), s.float(), mean, rstd, st["gamma"])
    ds = ds + st["ds"].float()
    return s, y.to(layer), mean, rstd, ds.to(stream), _plain_drop(st, ds, kept).to(layer), dgamma, dbeta


def _plain_sample(st):
    """In 64 bits: the numbers that decide lie next to borders."""
    z = st["logits"].double()
    n, v = z.shape
    z = torch.where(torch.isnan(z), torch.full((), -math.inf, device="cuda", dtype=F64), z)
    top = z.max(1, keepdim=True).values
    one = torch.ones((), device="cuda", dtype=F64)
    t = st["temperature"].double()[:, None] if st["temperature"] is not None else one.expand(n, 1)
    greedy = ~(t > 0)
    w = torch.where(z == top, one, torch.exp((z - top) / torch.where(greedy, one, t)))
    w = torch.where(z == -math.inf, 0 * one, w)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    ws = torch.gather(w, 1, order)
    keep = torch.ones_like(ws, dtype=torch.bool)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        keep &= (torch.arange(v, device="cuda")[None, :] < k) | (k <= 0)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        ws_k = torch.where(keep, ws, 0 * one)
        before = torch.cumsum(ws_k, 1) - ws_k
        keep &= (before < p * ws_k.sum(1, keepdim=True)) | (p >= 1)
        keep[:, 0] = True
    if st["min_p"] is not None:
        keep &= ws >= st["min_p"].double()[:, None].clamp(max=1.0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0 * one))
    cum = torch.cumsum(kept, 1)
    hit = (cum > st["u"].double()[:, None] * cum[:, -1:]) & (kept > 0)
    token = torch.where(greedy[:, 0], order[:, 0], hit.to(torch.uint8).argmax(1))
    return torch.where(top[:, 0] == -math.inf, torch.full((), -1, device="cuda", dtype=I64), token)


_PLAIN = {"layer_norm": _plain_layer_norm, "dropout": _plain_dropout, "residual_norm": _plain_residual_norm, "sample": _plain_sample}


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "sample":
        n, v = case["rows"], case["vocab"]
        params = sum(4 * n for k in ("temperature", "top_k", "top_p", "min_p") if case[k])
        return {"bytes": n * v * size[case["dtype"]] + 12 * n + params, "flops": 4.0 * n * v}
    n, c = case["rows"], case["cols"]
    e, b = n * c, size[case["dtype"]]
    draws = 30.0 * e if case.get("ratio", 0.0) > 0 else 0.0      # seven rounds for four elements
    if case["op"] == "dropout":
        return {"bytes": e * b * (5 if case["residual"] else 4) + 16, "flops": 2 * draws + 3.0 * e}
    if case["op"] == "layer_norm":
        o = size[case["out"]]
        fwd = {"bytes": e * (b + o) + 8 * c + 8 * n, "flops": 8.0 * e}
        if not case["backward"]:
            return fwd
        return {"bytes": fwd["bytes"] + e * (o + b + b) + 8 * n + 12 * c, "flops": fwd["flops"] + 14.0 * e}
    s = size[case["stream"]]
    # forward: x, residual -> s, y; backward: dy, ds, s -> dresidual, dx
    return {"bytes": e * (2 * b + 2 * s) + e * (2 * b + 3 * s) + 16 * n + 20 * c + 16, "flops": 2 * draws + 26.0 * e}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _exact_mask(case, st):
    """The mask in NumPy's unsigned integers, column blocks by row."""
    n, c = case["rows"], case["cols"]
    seed, offset = (int(v) for v in st["rng"].cpu())
    u32, u64 = np.uint32, np.uint64
    nb = (c + 3) // 4
    ctr = [np.tile(np.arange(nb, dtype=u32), n), np.repeat(np.arange(n, dtype=u32), nb),
           np.full(n * nb, offset & MASK, u32), np.full(n * nb, st["site"], u32)]
    key = [seed & MASK, seed >> 32 & MASK]
    for _ in range(ROUNDS):
        p0, p1 = ctr[0].astype(u64) * u64(M0), ctr[2].astype(u64) * u64(M1)
        hi0, hi1 = (p0 >> u64(32)).astype(u32), (p1 >> u64(32)).astype(u32)
        ctr = [hi1 ^ ctr[1] ^ u32(key[0]), p1.astype(u32), hi0 ^ ctr[3] ^ u32(key[1]), p0.astype(u32)]
        key = [(key[0] + W0) & MASK, (key[1] + W1) & MASK]
    words = np.stack(ctr, 1).reshape(n, nb * 4)[:, :c]
    return torch.from_numpy(words >= round(case["ratio"] * 2 ** 32)).cuda()


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "sample":
        return _exact_sample(case, st)
    d = lambda name: st[name].to(F64)
    if case["op"] == "layer_norm":
        x, gamma = d("x"), d("gamma")
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        r = (var + EPS) ** -0.5
        h = (x - mean) * r
        out = [h * gamma + d("beta"), mean[:, 0], r[:, 0]]
        if case["backward"]:
            dy = d("dy")
            q = dy * gamma
            out += [r * (q - q.mean(1, True) - h * (q * h).mean(1, True)), (h * dy).sum(0), dy.sum(0)]
        return tuple(out)
    scale = _exact_mask(case, st).to(F64) / (1.0 - case["ratio"])
    if case["op"] == "dropout":
        y = d("x") * scale
        return (y if st["residual"] is None else y + d("residual")), d("dy") * scale
    s = d("residual") + d("x") * scale
    # what is normalised is the sum as it is stored, after its roundings: the scale, the product, the sum, the stream's type
    product = (d("x") * scale.to(F32).to(F64)).to(F32).to(F64)
    kept = (d("residual") + product).to(F32).to(DT[case["stream"]]).to(F64)
    gamma, dy = d("gamma"), d("dy")
    var, mean = torch.var_mean(kept, 1, unbiased=False, keepdim=True)
    r = (var + EPS) ** -0.5
    h = (kept - mean) * r
    q = dy * gamma
    ds = r * (q - q.mean(1, True) - h * (q * h).mean(1, True)) + d("ds")
    return s, h * gamma + d("beta"), mean[:, 0], r[:, 0], ds, ds * scale, (h * dy).sum(0), dy.sum(0)


def _exact_sample(case, st):
    """Row by row on the host: filter the sorted tokens, walk the kept ones in the vocabulary's order."""
    z_all, u_all = st["logits"].float().cpu().numpy().astype(np.float64), st["u"].cpu().numpy().astype(np.float64)
    value = lambda name, i, none: none if st[name] is None else float(st[name][i])
    tokens = []
    for i, z in enumerate(z_all):
        ids = np.nonzero(z > -np.inf)[0]                       # (leaves NaN out)
        if len(ids) == 0:
            tokens.append(-1)
            continue
        t, best = value("temperature", i, 1.0), z[ids].max()
        if not t > 0:
            tokens.append(int(ids[np.argmax(z[ids])]))
            continue
        with np.errstate(invalid="ignore", over="ignore", under="ignore"):
            w = np.where(z[ids] == best, 1.0, np.exp((z[ids] - best) / t))
        down = np.argsort(-z[ids], kind="stable")
        k, p, least = int(value("top_k", i, 0)), value("top_p", i, 1.0), value("min_p", i, 0.0)
        if k > 0:
            down = down[:k]
        if p < 1:
            run = np.cumsum(w[down])
            down = down[:max(1, int(np.sum(run - w[down] < p * run[-1])))]
        down = np.sort(down[w[down] >= min(least, 1.0)])
        run = np.cumsum(w[down])
        tokens.append(int(ids[down[min(int(np.searchsorted(run, u_all[i] * run[-1], side="right")), len(down) - 1)]]))
    return torch.tensor(tokens)
