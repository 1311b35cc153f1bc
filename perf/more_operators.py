"""What a recurrent language model does from one token to the next, beside products, normalisation and sampling, as cases that can be timed and
compared.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass: in plain torch
where `own` is false, by the framework's entry points where it is true.  `work` counts the bytes and operations that the
pass cannot do without, `exact` has the same results from the definition in 64 bits.

Operators:
  scan     a gated linear recurrence over (T, B, D): kind sigmoid h_t = a h_{t-1} + (1 - a) x_t with a = 1 / (1 + exp(-gate)), kind decay
           h_t = gate_t h_{t-1} + x_t; y_t = h_t, the last state, and (backward) the gradients of gate, x and the first state.  Sequences may end
           early: behind their ends y and the gradients are 0 and the state stays
  embed    out[n] = scale * table[ids[n]], and the table's gradient scale * sum of the rows of dout that belong to each token; ids outside
           the table give rows of zeros and take no gradient
  adjust   logits before a token is drawn.  With c the number of times a token stands in a row's list, its prompt's tokens not counted for the last two:
           seen tokens z / repetition where z > 0 and z * repetition elsewhere, then - frequency * c - (presence if c > 0), then + its biases from a
           list, then -inf unless its bit of the row's mask is set
"""
import math

import numpy as np
import torch

own = False

F32, BF16, F64, I32, I64 = torch.float32, torch.bfloat16, torch.float64, torch.int32, torch.int64
DT = {"f32": F32, "bf16": BF16, "i32": I32, "i64": I64}
SIZE = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}


def listed():
    return [
        # One step of an answer: 128 sequences of the language model's width, latency counts.
        {"name": "scan_step_f32_128x650", "op": "scan", "steps": 1, "batch": 128, "cols": 650, "dtype": "f32", "out": "f32", "kind": "sigmoid",
         "backward": False, "lengths": False, "batch_first": False, "pad": 0},
        # The language model's window of 35 steps, a training step.
        {"name": "scan_f32_35x128x650", "op": "scan", "steps": 35, "batch": 128, "cols": 650, "dtype": "f32", "out": "f32", "kind": "sigmoid",
         "backward": True, "lengths": False, "batch_first": False, "pad": 0},
        # A wide layer in mixed precision, sequences of 2048 steps.
        {"name": "scan_bf16_2048x8x4096", "op": "scan", "steps": 2048, "batch": 8, "cols": 4096, "dtype": "bf16", "out": "bf16", "kind": "sigmoid",
         "backward": True, "lengths": False, "batch_first": True, "pad": 0},
        # One very long sequence with given decays, a few of them 0 where another document begins.
        {"name": "scan_bf16_65536x1x1024", "op": "scan", "steps": 65536, "batch": 1, "cols": 1024, "dtype": "bf16", "out": "bf16", "kind": "decay",
         "backward": True, "lengths": False, "batch_first": False, "pad": 0},
        # A ragged batch of odd sizes inside wider rows.
        {"name": "scan_f32_777x5x1001", "op": "scan", "steps": 777, "batch": 5, "cols": 1001, "dtype": "f32", "out": "f32", "kind": "decay",
         "backward": True, "lengths": True, "batch_first": False, "pad": 3},
        # The language model's embeddings and their gradient.
        {"name": "embed_f32_4480x650_v10000", "op": "embed", "tokens": 4480, "cols": 650, "vocab": 10000, "table": "f32", "out": "f32", "ids": "i64", "pad": 0},
        # A large vocabulary in mixed precision, tokens as frequent as words are.
        {"name": "embed_bf16_65536x1024_v131072", "op": "embed", "tokens": 65536, "cols": 1024, "vocab": 131072, "table": "bf16", "out": "bf16", "ids": "i64", "pad": 0},
        # More tokens than the table has rows: bytes, or classes, of odd width.
        {"name": "embed_f32_100003x333_v257", "op": "embed", "tokens": 100003, "cols": 333, "vocab": 257, "table": "f32", "out": "f32", "ids": "i32", "pad": 3},
        # The language model answers: penalties for what the last window holds.
        {"name": "adjust_f32_128x10000", "op": "adjust", "rows": 128, "vocab": 10000, "dtype": "f32", "out": "f32", "history": 35, "prompt": True,
         "repetition": True, "frequency": True, "presence": True, "biases": 0, "masked": 0.0, "ids": "i64", "pad": 0},
        # A single request with a large vocabulary and a grammar.
        {"name": "adjust_bf16_1x131072", "op": "adjust", "rows": 1, "vocab": 131072, "dtype": "bf16", "out": "f32", "history": 2048, "prompt": True,
         "repetition": True, "frequency": False, "presence": False, "biases": 16, "masked": 0.99, "ids": "i64", "pad": 0},
        # A full batch with long texts, everything on.
        {"name": "adjust_f32_256x131072", "op": "adjust", "rows": 256, "vocab": 131072, "dtype": "f32", "out": "f32", "history": 8192, "prompt": True,
         "repetition": True, "frequency": True, "presence": True, "biases": 300, "masked": 0.5, "ids": "i32", "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over the logarithm of its range: a third as drawn, a third multiples of 8, a third of 64."""
    n, step = _log(rng, lo, hi), rng.choice((1, 8, 64))
    return max(lo, min(hi, (n + step - 1) // step * step))


def draw(rng):
    op = rng.choice(("scan", "scan", "scan", "embed", "embed", "adjust", "adjust"))
    dtype, pad = rng.choice(("f32", "bf16")), rng.choice((0, 0, 3, 8))
    out = rng.choice((dtype, dtype, "f32"))
    if op == "scan":
        cols = _size(rng, 16, 8192)
        batch = _log(rng, 1, min(256, 2 ** 20 // cols))
        most = 2 ** 30 // (6 * SIZE[dtype] + 2 * SIZE[out])      # elements, so that a pass moves no more than the largest listed one
        steps = _log(rng, 1, max(1, min(65536, most // (cols * batch))))
        return {"op": op, "steps": steps, "batch": batch, "cols": cols, "dtype": dtype, "out": out,
                "kind": rng.choice(("sigmoid", "decay")), "backward": rng.random() < 0.7, "lengths": rng.random() < 0.4,
                "batch_first": rng.random() < 0.5, "pad": pad}
    if op == "embed":
        cols = _size(rng, 4, 4096)
        return {"op": op, "tokens": min(_log(rng, 1, 131072), 2 ** 27 // cols // SIZE[out]), "cols": cols, "vocab": min(_size(rng, 2, 131072), 15 * 2 ** 23 // cols),
                "table": dtype, "out": out, "ids": rng.choice(("i32", "i64")), "pad": pad}
    on = lambda share: rng.random() < share
    history, biases, masked = rng.choice((0, _log(rng, 1, 8192), _log(rng, 1, 8192))), rng.choice((0, 0, _log(rng, 1, 300))), rng.choice((0.0, 0.5, 0.999))
    frequency, presence = on(0.5), on(0.5)
    # (a call that asks for something: the repetition where nothing else reads the lists, a mask where there are no lists and no biases)
    return {"op": op, "rows": _log(rng, 1, 240), "vocab": _size(rng, 2, 131072), "dtype": dtype, "out": out,
            "history": history, "prompt": on(0.5), "repetition": on(0.7) or not (frequency or presence), "frequency": frequency, "presence": presence,
            "biases": biases, "masked": masked if history or biases or masked > 0 else 0.5, "ids": rng.choice(("i32", "i64")), "pad": pad}


# ---- what a program holds before the call -----------------------------------------------------------------------
def _words(gen, n, vocab):
    """Tokens as frequent as words are: the k-th most frequent about one in k, in an order of the table's own."""
    rank = torch.exp(torch.rand(n, generator=gen, device="cuda", dtype=F64) * math.log(vocab + 1)).long() - 1
    return torch.randperm(vocab, generator=gen, device="cuda")[rank.clamp_(0, vocab - 1)]


def _steps(case, width, dtype, batch_first):
    """Memory for (T, B, width) values, rows `pad` elements longer, time or batch outermost."""
    t, b, w = case["steps"], case["batch"], width + case["pad"]
    buf = torch.empty((b, t, w) if batch_first else (t, b, w), device="cuda", dtype=DT[dtype])
    return (buf.transpose(0, 1) if batch_first else buf)[:, :, :width]


def _prepare_scan(case, gen, st):
    t, b, c = case["steps"], case["batch"], case["cols"]
    # gates and inputs are the halves of one product's result
    z = _steps(case, 2 * c, case["dtype"], case["batch_first"])
    st["gate"], st["x"] = z[:, :, :c], z[:, :, c:]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    g = normal(t, b, c) * 1.5 + 2.0
    if case["kind"] == "decay":
        g = torch.where(torch.rand(t, b, 1, generator=gen, device="cuda") < 1 / 512, torch.zeros((), device="cuda"), torch.sigmoid(g + 1.0))
    st["gate"].copy_(g)
    st["x"].copy_(normal(t, b, c))
    st["h0"] = normal(b, c)
    st["lengths"] = torch.randint(0, t + 1, (b,), generator=gen, device="cuda") if case["lengths"] else None
    if case["backward"]:
        st["dy"] = _steps(case, c, case["out"], case["batch_first"])
        st["dy"].copy_(normal(t, b, c) * 1e-2)
        st["dh_last"] = normal(b, c) * 1e-2
    if own:
        from paper_1908_00213_amd import binding as B
        st["y"], st["h_last"] = _steps(case, c, case["out"], case["batch_first"]), torch.empty(b, c, device="cuda")
        st["ws"] = torch.empty(max(256, B.gated_scan_workspace_bytes(st["gate"])), device="cuda", dtype=torch.uint8)
        st["states"] = None
        if case["backward"]:
            dz = _steps(case, 2 * c, case["dtype"], case["batch_first"])
            st["dgate"], st["dx"], st["dh0"] = dz[:, :, :c], dz[:, :, c:], torch.empty(b, c, device="cuda")
            st["states"] = torch.empty(B.gated_scan_states_shape(t, b, c), device="cuda")


def _prepare_embed(case, gen, st):
    n, c, v, pad = case["tokens"], case["cols"], case["vocab"], case["pad"]
    st["scale"] = math.sqrt(c)
    ids = _words(gen, n, v)
    # (padding of batches: a token in a hundred is none)
    st["ids"] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.01, torch.full((), -1, device="cuda"), ids).to(DT[case["ids"]])
    st["table"] = (torch.randn(v, c + pad, generator=gen, device="cuda") / math.sqrt(c)).to(DT[case["table"]])[:, :c]
    st["dout"] = (torch.randn(n, c + pad, generator=gen, device="cuda") * 1e-2).to(DT[case["out"]])[:, :c]
    if own:
        from paper_1908_00213_amd import binding as B
        st["out"] = torch.empty(n, c + pad, device="cuda", dtype=DT[case["out"]])[:, :c]
        st["dtable"] = torch.empty(v, c + pad, device="cuda")[:, :c]
        st["ws"] = torch.empty(max(256, B.embed_sorted_workspace_bytes(st["ids"], st["dtable"])), device="cuda", dtype=torch.uint8)


def _prepare_adjust(case, gen, st):
    n, v, l, m = case["rows"], case["vocab"], case["history"], case["biases"]
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")
    st["logits"] = (torch.randn(n, v + case["pad"], generator=gen, device="cuda") * 2.5).to(DT[case["dtype"]])[:, :v]
    st["tokens"] = _words(gen, n * l, v).view(n, l).to(DT[case["ids"]]) if l else None
    st["lengths"] = torch.randint(0, l + 1, (n,), generator=gen, device="cuda") if l else None
    st["prompt"] = (st["lengths"] * uniform(n)).long() if l and case["prompt"] else None
    st["repetition"] = 1.0 + 0.3 * uniform(n) if case["repetition"] else None
    st["frequency"] = 0.5 * uniform(n) if case["frequency"] else None
    st["presence"] = 0.5 * uniform(n) if case["presence"] else None
    st["bias_ids"] = torch.randint(0, v, (n, m), generator=gen, device="cuda").to(DT[case["ids"]]) if m else None
    st["bias"] = torch.randn(n, m, generator=gen, device="cuda") * 5 if m else None
    st["allowed"] = None
    if case["masked"] > 0:
        bits = (uniform(n, (v + 31) // 32, 32) >= case["masked"]).long()
        word = (bits << torch.arange(32, device="cuda")).sum(-1)
        st["allowed"] = torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(I32)
    if own:
        st["out"] = torch.empty(n, v + case["pad"], device="cuda", dtype=DT[case["out"]])[:, :v]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    {"scan": _prepare_scan, "embed": _prepare_embed, "adjust": _prepare_adjust}[case["op"]](case, gen, st)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _PLAIN[st["case"]["op"]](st)


def _run_own(st):
    from paper_1908_00213_amd import binding as B
    case = st["case"]
    op = case["op"]
    if op == "embed":
        B.embed_scaled_fwd(st["table"], st["ids"], st["out"], st["scale"])
        B.embed_sorted_bwd(st["ids"], st["dout"], st["dtable"], st["scale"], ws=st["ws"])
        return st["out"], st["dtable"]
    if op == "adjust":
        return B.logits_adjust(st["logits"], st["out"], tokens=st["tokens"], lengths=st["lengths"], prompt=st["prompt"], repetition=st["repetition"],
                               frequency=st["frequency"], presence=st["presence"], bias_ids=st["bias_ids"], bias=st["bias"], allowed=st["allowed"])
    B.gated_scan_fwd(st["gate"], st["x"], st["y"], h0=st["h0"], h_last=st["h_last"], states=st["states"], lengths=st["lengths"], kind=case["kind"], ws=st["ws"])
    if not case["backward"]:
        return st["y"], st["h_last"]
    B.gated_scan_bwd(st["gate"], st["x"], st["states"], st["dy"], st["dgate"], st["dx"], dh_last=st["dh_last"], dh0=st["dh0"], lengths=st["lengths"],
                     kind=case["kind"], ws=st["ws"])
    return st["y"], st["h_last"], st["dgate"], st["dx"], st["dh0"]


def _scan(a, u, first):
    """h_t = a_t h_{t-1} + u_t from h_{-1} = first, all steps at once: after a round with distance s, a and u span 2 s steps."""
    u[0] += a[0] * first
    s, n = 1, len(a)
    while s < n:
        u = torch.cat([u[:s], a[s:] * u[:-s] + u[s:]])
        a = torch.cat([a[:s], a[s:] * a[:-s]])
        s *= 2
    return u


def _plain_scan(st):
    case = st["case"]
    t = case["steps"]
    g, x = st["gate"].float(), st["x"].float()
    sigmoid = case["kind"] == "sigmoid"
    a = 1.0 / (1.0 + torch.exp(-g)) if sigmoid else g
    rest = 1.0 / (1.0 + torch.exp(g)) if sigmoid else None
    u = rest * x if sigmoid else x.clone()
    if st["lengths"] is not None:
        live = (torch.arange(t, device="cuda")[:, None] < st["lengths"][None, :])[:, :, None]
        zero, one = torch.zeros((), device="cuda"), torch.ones((), device="cuda")
        u, ah = torch.where(live, u, zero), torch.where(live, a, one)
    else:
        live, ah = None, a
    h = _scan(ah, u, st["h0"])
    keep = lambda v: v if live is None else torch.where(live, v, zero)
    y, last = keep(h).to(DT[case["out"]]), h[-1].clone()
    if not case["backward"]:
        return y, last
    dy = keep(st["dy"].float())
    # G_t = dy_t + a_{t+1} G_{t+1}, backwards in time
    back = torch.cat([torch.ones_like(ah[:1]), ah[1:].flip(0)])
    G = _scan(back, dy.flip(0).clone(), st["dh_last"]).flip(0)
    before = torch.cat([st["h0"][None], h[:-1]])
    dt = DT[case["dtype"]]
    dx = keep(G * rest if sigmoid else G).to(dt)
    dg = keep(G * (before - x) * a * rest if sigmoid else G * before).to(dt)
    return y, last, dg, dx, ah[0] * G[0]


def _plain_embed(st):
    case = st["case"]
    v = case["vocab"]
    ids = st["ids"].long()
    ok = ((ids >= 0) & (ids < v))[:, None]
    at = ids.clamp(0, v - 1)
    zero = torch.zeros((), device="cuda")
    out = torch.where(ok, st["table"][at].float() * st["scale"], zero).to(DT[case["out"]])
    rows = torch.where(ok, st["dout"].float(), zero)
    dtable = torch.zeros(v, case["cols"], device="cuda").index_add_(0, at, rows) * st["scale"]
    return out, dtable


def _plain_adjust(st):
    case = st["case"]
    n, v = case["rows"], case["vocab"]
    z = st["logits"].float()
    if st["tokens"] is not None:
        tok = st["tokens"].long()
        place = torch.arange(tok.shape[1], device="cuda")[None, :]
        live = place < st["lengths"][:, None]
        mine = live if st["prompt"] is None else live & (place >= st["prompt"][:, None])
        count = lambda which: torch.zeros(n, v, device="cuda").scatter_add_(1, tok, which.float())
        seen, c = count(live) > 0, count(mine)
        if st["repetition"] is not None:
            r = st["repetition"][:, None]
            z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
        if st["frequency"] is not None:
            z = z - st["frequency"][:, None] * c
        if st["presence"] is not None:
            z = z - st["presence"][:, None] * (c > 0)
    if st["bias"] is not None:
        z = z + torch.zeros(n, v, device="cuda").scatter_add_(1, st["bias_ids"].long(), st["bias"])
    if st["allowed"] is not None:
        bits = (st["allowed"].long()[:, :, None] >> torch.arange(32, device="cuda")) & 1
        z = torch.where(bits.reshape(n, -1)[:, :v] > 0, z, torch.full((), -math.inf, device="cuda"))
    return z.to(DT[case["out"]])


_PLAIN = {"scan": _plain_scan, "embed": _plain_embed, "adjust": _plain_adjust}


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def _distinct(n, v):
    """How many different tokens n draws of `_words` hold, on average."""
    p = np.diff(np.log(np.arange(1, v + 2))) / math.log(v + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    if case["op"] == "scan":
        b, c = case["batch"], case["cols"]
        e, s, o = case["steps"] * b * c, SIZE[case["dtype"]], SIZE[case["out"]]
        bytes_, flops = e * (2 * s + o) + 8 * b * c, 6.0 * e
        if case["backward"]:
            bytes_, flops = bytes_ + e * (4 * s + o) + 8 * b * c, flops + 16.0 * e
        return {"bytes": bytes_ + (8 * b if case["lengths"] else 0), "flops": flops}
    if case["op"] == "embed":
        n, c, v = case["tokens"], case["cols"], case["vocab"]
        return {"bytes": 2 * n * SIZE[case["ids"]] + _distinct(n, v) * c * SIZE[case["table"]] + 2 * n * c * SIZE[case["out"]] + 4 * v * c, "flops": 3.0 * n * c}
    n, v = case["rows"], case["vocab"]
    lists = n * (case["history"] / 2 * SIZE[case["ids"]] + 24 + case["biases"] * (SIZE[case["ids"]] + 4))
    return {"bytes": n * v * (SIZE[case["dtype"]] + SIZE[case["out"]]) + (n * v / 8 if case["masked"] > 0 else 0) + lists, "flops": 4.0 * n * v}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"scan": _exact_scan, "embed": _exact_embed, "adjust": _exact_adjust}[case["op"]](case, st)


def _exact_scan(case, st):
    """Step by step."""
    t = case["steps"]
    sigmoid = case["kind"] == "sigmoid"
    ends = None if st["lengths"] is None else st["lengths"]
    gates = st["gate"].contiguous().to(F64)
    a = torch.sigmoid(gates) if sigmoid else gates
    rest = torch.sigmoid(-gates) if sigmoid else None
    x = st["x"].contiguous().to(F64)
    h = st["h0"].to(F64)
    before, y = torch.empty_like(a), torch.empty_like(a)
    for i in range(t):
        before[i] = h
        new = a[i] * h + (rest[i] * x[i] if sigmoid else x[i])
        if ends is None:
            h = new
            y[i] = h
        else:
            on = (i < ends)[:, None]
            h = torch.where(on, new, h)
            y[i] = h * on
    if not case["backward"]:
        return y, h
    dy = st["dy"].contiguous().to(F64)
    G, dx, dg = st["dh_last"].to(F64), torch.empty_like(a), torch.empty_like(a)
    for i in range(t - 1, -1, -1):
        here = G + dy[i]
        back = a[i] * here
        if ends is not None:
            on = (i < ends)[:, None]
            back, here = torch.where(on, back, G), here * on
        dx[i] = here
        G = back
    if sigmoid:
        dg = dx * (before - x) * a * rest
        dx = dx * rest
    else:
        dg = dx * before
    return y, h, dg, dx, G


def _exact_embed(case, st):
    """Rows in the order of their tokens, summed between the places where another token begins."""
    v, c = case["vocab"], case["cols"]
    ids = st["ids"].cpu().numpy().astype(np.int64)
    good = (ids >= 0) & (ids < v)
    out = torch.zeros(len(ids), c, device="cuda", dtype=F64)
    at = torch.from_numpy(np.nonzero(good)[0]).cuda()
    out[at] = st["table"][torch.from_numpy(ids[good]).cuda()].to(F64) * st["scale"]
    order = np.argsort(np.where(good, ids, v), kind="stable")[:int(good.sum())]
    dtable = torch.zeros(v, c, device="cuda", dtype=F64)
    if len(order):
        names, first, counts = np.unique(ids[order], return_index=True, return_counts=True)
        rows = st["dout"][torch.from_numpy(order).cuda()].to(F64)
        for lo in range(0, c, 64):                       # running sums of a few columns at a time
            run_ = torch.cumsum(rows[:, lo:lo + 64], 0)
            end = run_[torch.from_numpy(first + counts - 1).cuda()]
            begin = torch.cat([torch.zeros_like(end[:1]), end[:-1]])
            dtable[torch.from_numpy(names).cuda(), lo:lo + 64] = (end - begin) * st["scale"]
    return out, dtable


def _exact_adjust(case, st):
    """Row by row on the host."""
    host = lambda name: None if st[name] is None else st[name].cpu().numpy()
    z_all = st["logits"].float().cpu().numpy().astype(np.float64)
    tokens, lengths, prompt, ids, bias, allowed = (host(k) for k in ("tokens", "lengths", "prompt", "bias_ids", "bias", "allowed"))
    rep, freq, pres = (host(k) for k in ("repetition", "frequency", "presence"))
    for i, z in enumerate(z_all):
        if tokens is not None:
            row = tokens[i, :lengths[i]].astype(np.int64)
            mine = row if prompt is None else row[prompt[i]:]
            if rep is not None:
                s = np.unique(row)
                z[s] = np.where(z[s] > 0, z[s] / np.float64(rep[i]), z[s] * np.float64(rep[i]))
            names, c = np.unique(mine, return_counts=True)
            if freq is not None:
                z[names] -= np.float64(freq[i]) * c
            if pres is not None:
                z[names] -= np.float64(pres[i])
        if bias is not None:
            np.add.at(z, ids[i].astype(np.int64), bias[i].astype(np.float64))
        if allowed is not None:
            bits = np.unpackbits(np.ascontiguousarray(allowed[i]).view(np.uint8), bitorder="little")[:len(z)]
            z[bits == 0] = -np.inf
    return torch.from_numpy(z_all)
