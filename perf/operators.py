"""The operators that train and serve a mixture of heads outside the renderer, as a program calls them.

A case names one operator and its sizes:

  sort     (sample, slot) pairs sorted stably by head, and the samples' rows brought into that order; with
           train also the gradient of that, a sum over each sample's pairs.  A pair may have no head.
  join     each sample's rows brought back and summed with their weights, and the gradients of that
  forward  every head's linear layer on its rows, with bias and ReLU
  backward the gradients of that layer: inputs, weights, biases
  adamw    one AdamW step over many tensors, moments in 32 bits, or in e4m3 with a scale for 256 values

Each has a plain form (elementary torch operations in float32) and, where own is true, the calls of
paper_2011_12490_amd.heads.  exact() computes the same in float64.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
BLOCK = 256              # values of an 8-bit moment that share a scale
FP8 = torch.float8_e4m3fn
FP8_MAX = 448.0
FP8_LEAST = 2.0 ** -9    # smallest positive e4m3
SCALE_LEAST = 2.0 ** -120
LR, BETA1, BETA2, EPS, DECAY = 5e-4, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # eight samples of a probe or a serving loop: launches and latency
        _sort("sort_few", 8, 2, 16, 256, "bf16", 0.0, False),
        # the largest batch that is brought into the heads' order, with its gradient; some pairs masked
        _sort("sort_large", 131072, 4, 64, 1024, "bf16", 0.05, True),
        # a training batch of 512 rays of 128 samples, each through its two nearest heads: density and colour come back
        _join("join_batch", 512 * 128, 2, 16, 4, "fp32", 0.1),
        # wide rows through eight of 64 heads
        _join("join_large", 16384, 8, 64, 2048, "bf16", 0.0),
        # single samples through wide heads: the weights are what is read
        _linear("forward_few", "forward", 16, 16, 1024, 4096, "bf16", True),
        # the skip layer of 8x256 heads ([gamma(x); h]: 63 + 256 inputs) on a ragged batch
        _linear("forward_skip", "forward", 262139, 16, 319, 256, "bf16", True),
        # wide heads at a large batch
        _linear("forward_wide", "forward", 32768, 8, 2048, 4096, "bf16", True),
        # the first layer of 8x128 heads in float32 (63 inputs)
        _linear("backward_first_fp32", "backward", 98301, 16, 63, 128, "fp32", True),
        # a hidden layer of 8x128 heads, two heads a sample
        _linear("backward_hidden", "backward", 131072, 16, 128, 128, "bf16", True),
        # wide heads, both gradients
        _linear("backward_wide", "backward", 16384, 8, 2048, 4096, "bf16", False),
        # the tensors of 16 heads of 8x128, bf16 copies kept for the matrix units
        _adamw("adamw_heads", 22, 2_400_000, 32, "fp32", "fp32", True),
        # wide heads with their moments in 8 bits
        _adamw("adamw_large", 96, 200_000_000, 8, "fp32", "bf16", False),
    ]


def _sort(name, tokens, top_k, heads, dim, dtype, dropped, train):
    return _named(name, call="sort", tokens=tokens, top_k=top_k, heads=heads, dim=dim, dtype=dtype, dropped=dropped, train=train)


def _join(name, tokens, top_k, heads, dim, dtype, dropped):
    return _named(name, call="join", tokens=tokens, top_k=top_k, heads=heads, dim=dim, dtype=dtype, dropped=dropped)


def _linear(name, call, rows, heads, fan_in, fan_out, dtype, relu, dropped=0.0):
    return _named(name, call=call, rows=rows, heads=heads, fan_in=fan_in, fan_out=fan_out, dtype=dtype, relu=relu, dropped=dropped)


def _adamw(name, tensors, values, bits, dtype, grad, copy):
    return _named(name, call="adamw", tensors=tensors, values=values, bits=bits, dtype=dtype, grad=grad, copy=copy)


def _named(name, **case):
    return dict(case, name=name) if name else case


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["sort", "join", "forward", "forward", "backward", "backward", "adamw"])
    while True:
        dtype = rng.choice(["fp32", "bf16"])
        heads = _spread(rng, 2, 128)
        dropped = rng.choice([0.0, 0.0, 0.03, 0.3])
        if call in ("sort", "join"):
            tokens, top_k = _spread(rng, 1, 131072), rng.randint(1, min(8, heads))
            dim = _spread(rng, 3, 2048)
            if tokens * top_k * dim * BYTES[dtype] > 1 << 29:
                continue
            if call == "sort":
                return _sort(None, tokens, top_k, heads, dim, dtype, dropped, rng.random() < 0.5)
            return _join(None, tokens, top_k, heads, dim, dtype, dropped)
        if call in ("forward", "backward"):
            # odd widths are those of encodings and skip inputs
            fan_in = rng.choice([27, 39, 63, 64, 91, 128, 155, 191, 256, 283, 319, _spread(rng, 16, 2048), 64 * rng.randint(1, 32)])
            fan_out = rng.choice([1, 3, 4, 32, 64, 64, 128, 128, 256, 256, _spread(rng, 16, 4096), 64 * rng.randint(1, 64)])
            rows = _spread(rng, 1, 262144)
            cost = 2.0 * rows * fan_in * fan_out * (2 if call == "backward" else 1) * (2 if dtype == "fp32" else 1)
            if cost > 4e11 or rows * (fan_in + fan_out) > 1 << 28 or heads * fan_in * fan_out > 1 << 26:
                continue
            return _linear(None, call, rows, heads, fan_in, fan_out, dtype, rng.random() < 0.6, dropped)
        return _adamw(None, rng.randint(1, 300), _spread(rng, 20_000, 150_000_000), rng.choice([8, 32]), dtype,
                      rng.choice(["fp32", "bf16"]), dtype == "fp32" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------

def _shares(rng, heads):
    """How often each head is taken: far from even, as cells of a scene are."""
    p = rng.gamma(1.5, 1.0, heads) + 0.02
    return p / p.sum()


def _ids(case, g, rng):
    """Each sample's top_k different heads; a masked pair has -1."""
    T, k, K = case["tokens"], case["top_k"], case["heads"]
    liking = torch.from_numpy(np.log(_shares(rng, K))).float().cuda()
    noise = -torch.log(-torch.log(torch.rand(T, K, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7)))
    score, ids = torch.topk(liking + noise, k, dim=1)
    if case["dropped"]:
        ids = torch.where(torch.rand(T, k, generator=g, device="cuda") < case["dropped"], -1, ids)
    return ids.int().contiguous(), torch.softmax(score, dim=1).contiguous()


def _order(ids, heads):
    """offsets, pair, row of the stable order by head, pairs without a head last (their row is -1 - place)."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < heads), flat, heads)
    pair = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[pair], torch.arange(heads + 1, device=ids.device))
    place = torch.empty_like(pair)
    place[pair] = torch.arange(pair.numel(), device=ids.device)
    row = torch.where(key < heads, place, -1 - place)
    return offsets.int(), pair.int(), row.int().reshape(ids.shape)


def _sizes(case):
    """Values of each tensor: a few large ones, many small ones, odd counts, as weights and biases are."""
    rng = np.random.default_rng(case["tensors"] * 7919 + case["values"] % 7919)
    share = np.exp(rng.uniform(0.0, 5.0, case["tensors"]))
    return [int(n) for n in np.maximum(1, share / share.sum() * case["values"]).astype(np.int64)]


def _starts(sizes):
    """Where each tensor starts in a buffer of them all: at a multiple of BLOCK."""
    ends = np.cumsum([-(-n // BLOCK) * BLOCK for n in sizes])
    return [0] + [int(e) for e in ends]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    call = case["call"]
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    if call in ("sort", "join"):
        dtype = TYPES[case["dtype"]]
        ids, weights = _ids(case, g, rng)
        pairs = ids.numel()
        s = {"case": case, "ids": ids}
        if call == "sort":
            s["x"] = rand(case["tokens"], case["dim"]).to(dtype)
            s["grad"] = rand(pairs, case["dim"]).to(dtype) if case["train"] else None
            return s
        s["order"] = _order(ids, case["heads"])
        s["rows"], s["weights"] = rand(pairs, case["dim"]).to(dtype), weights
        s["grad"] = (0.1 * rand(case["tokens"], case["dim"])).to(dtype)
        if own:
            from paper_2011_12490_amd import heads
            s["routing"] = heads.Routing(*s["order"], case["heads"])
        return s
    if call in ("forward", "backward"):
        dtype = TYPES[case["dtype"]]
        R, K, I, O = (case[n] for n in ("rows", "heads", "fan_in", "fan_out"))
        counts = rng.multinomial(R - int(R * case["dropped"]), _shares(rng, K))
        s = {"case": case, "counts": [int(n) for n in counts],
             "offsets": torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda"),
             "x": rand(R, I).clamp_min(0).to(dtype), "w": (rand(K, O, I) * (2.0 / I) ** 0.5).to(dtype), "b": 0.1 * rand(K, O)}
        if call == "backward":
            s["grad"] = (0.1 * rand(R, O)).to(dtype)
            s["y"] = rand(R, O).clamp_min(0).to(dtype) if case["relu"] else None  # the layer's output, as kept for this
        return s
    sizes = _sizes(case)
    starts, total = _starts(sizes), _starts(sizes)[-1]
    used = torch.zeros(total + 1, device="cuda", dtype=torch.int32)
    used[torch.tensor(starts[:-1], device="cuda")] += 1
    used[torch.tensor(starts[:-1], device="cuda") + torch.tensor(sizes, device="cuda")] -= 1
    used = (torch.cumsum(used, 0)[:-1] > 0).float()
    # a tensor's gradients have a size of their own, and some of its rows got none
    size = torch.exp(rand(total // BLOCK) * 1.5 - 8).repeat_interleave(BLOCK)
    size = size * (torch.rand(total // BLOCK, generator=g, device="cuda") > 0.05).repeat_interleave(BLOCK) * used
    m, root = rand(total) * size * 0.3, (rand(total).abs() * 0.5 + 0.7) * size
    s = {"case": case, "step": 100, "scale": torch.rand(1, generator=g, device="cuda") * 0.5 + 0.5,
         "p": (0.05 * rand(total) * used).to(TYPES[case["dtype"]]), "g": (rand(total) * size).to(TYPES[case["grad"]]),
         "copy": torch.zeros(total, device="cuda", dtype=torch.bfloat16) if case["copy"] else None}
    del used, size
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to8(m, False)
        s["v"], s["v_scale"] = _to8(root, True)
    else:
        s["m"], s["v"] = m, root * root
        s["m_scale"] = s["v_scale"] = None
    if own:
        from paper_2011_12490_amd import heads
        cut = lambda t: None if t is None else [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        scales = lambda t: None if t is None else [t[a // BLOCK:b // BLOCK] for a, b in zip(starts, starts[1:])]  # noqa: E731
        s["optimizer"] = heads.AdamW(cut(s["p"]), cut(s["g"]), m=cut(s["m"]), v=cut(s["v"]), m_scale=scales(s["m_scale"]),
                                     v_scale=scales(s["v_scale"]), copies=cut(s["copy"]), lr=LR, betas=(BETA1, BETA2), eps=EPS,
                                     weight_decay=DECAY, state_bits=case["bits"])
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s["case"], s)


def _run_own(case, s):
    from paper_2011_12490_amd import heads
    call = case["call"]
    if call == "sort":
        r = heads.route(s["ids"], case["heads"])
        rows = heads.dispatch(s["x"], r)
        dx = heads.dispatch_backward(s["grad"], r) if case["train"] else None
        return {"offsets": r.offsets, "pair": r.pair, "row": r.row, "rows": rows, "dx": dx}
    if call == "join":
        y = heads.combine(s["rows"], s["routing"], s["weights"])
        drows, dweights = heads.combine_backward(s["grad"], s["rows"], s["routing"], s["weights"])
        return {"y": y, "drows": drows, "dweights": dweights}
    if call == "forward":
        return {"y": heads.linear(s["x"], s["w"], s["b"], s["offsets"], relu=case["relu"])}
    if call == "backward":
        dx, dw, db = heads.linear_backward(s["grad"], s["x"], s["w"], s["offsets"], y=s["y"])
        return {"dx": dx, "dw": dw, "db": db}
    s["step"] += 1
    s["optimizer"].step(s["step"], grad_scale=s["scale"])
    return _state(s)


def _state(s):
    return {n: s[n] for n in ("p", "copy", "m", "v", "m_scale", "v_scale")}


def _run_plain(case, s):
    call = case["call"]
    if call == "sort":
        offsets, pair, row = _order(s["ids"], case["heads"])
        k = case["top_k"]
        headed = (torch.arange(pair.numel(), device="cuda") < offsets[-1])[:, None]
        rows = torch.where(headed, s["x"][pair.long() // k], torch.zeros((), dtype=s["x"].dtype, device="cuda"))
        dx = _gather_sum(s["grad"], row, None) if case["train"] else None
        return {"offsets": offsets, "pair": pair, "row": row, "rows": rows, "dx": dx}
    if call == "join":
        offsets, pair, row = s["order"]
        y = _gather_sum(s["rows"], row, s["weights"])
        grad, k = s["grad"].float(), case["top_k"]
        at, with_head = _places(row)
        dweights = (s["rows"][at].float().reshape(*row.shape, -1) * grad[:, None]).sum(-1) * with_head
        of_row = pair.long()
        weight = (s["weights"] * with_head).reshape(-1)[of_row]
        drows = (grad[of_row // k] * weight[:, None]).to(s["rows"].dtype)
        return {"y": y, "drows": drows, "dweights": dweights}
    if call == "forward":
        # a head's rows lie one after another, so each head is one product; the counts are known on the host here
        x, w, b = s["x"].float(), s["w"].float(), s["b"]
        headed = sum(s["counts"])
        parts = torch.split(x[:headed], s["counts"])
        y = torch.cat([p @ w[h].T + b[h] for h, p in enumerate(parts)] + [x.new_zeros(x.shape[0] - headed, w.shape[1])])
        return {"y": (y.clamp_min(0) if case["relu"] else y).to(s["x"].dtype)}
    if call == "backward":
        x, w, dz = s["x"].float(), s["w"].float(), s["grad"].float()
        if case["relu"]:
            dz = dz * (s["y"] > 0)
        headed = sum(s["counts"])
        xs, zs = torch.split(x[:headed], s["counts"]), torch.split(dz[:headed], s["counts"])
        dx = torch.cat([z @ w[h] for h, z in enumerate(zs)] + [x.new_zeros(x.shape[0] - headed, x.shape[1])])
        dw = torch.stack([z.T @ p for z, p in zip(zs, xs)])
        db = torch.stack([z.sum(0) for z in zs])
        return {"dx": dx.to(s["x"].dtype), "dw": dw, "db": db}
    s["step"] += 1
    t = s["step"]
    decay, rate, root2 = 1.0 - LR * DECAY, LR / (1.0 - BETA1 ** t), 1.0 / math.sqrt(1.0 - BETA2 ** t)
    m, v = (s["m"], s["v"]) if case["bits"] == 32 else (_from8(s["m"], s["m_scale"]), _from8(s["v"], s["v_scale"]).square())
    grad = s["g"].float() * s["scale"]
    m = m * BETA1 + grad * (1.0 - BETA1)
    v = v * BETA2 + grad * grad * (1.0 - BETA2)
    root = torch.sqrt(v)
    p = s["p"].float() * decay - m / (root * root2 + EPS) * rate
    s["p"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for name, new, is_root in (("m", m, False), ("v", root, True)):
            codes, scale = _to8(new, is_root)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    return _state(s)


def _places(row):
    """The place of every pair, and 1 where it has a head."""
    row = row.long()
    return torch.where(row < 0, -1 - row, row).reshape(-1), (row >= 0).float()


def _gather_sum(rows, row, weights):
    at, with_head = _places(row)
    factor = with_head if weights is None else with_head * weights
    return (rows[at].float().reshape(*row.shape, -1) * factor[..., None]).sum(1).to(rows.dtype)


def _to8(x, is_root):
    """x (a multiple of BLOCK values) as e4m3 and a scale for each block: its largest value becomes FP8_MAX.  A root
    that is not zero keeps the smallest code at least, since it is divided by."""
    x = x.reshape(-1, BLOCK)
    scale = (x.abs().amax(1, keepdim=True) * x.new_tensor(1.0 / FP8_MAX)).clamp_min(SCALE_LEAST)
    scaled = (x * scale.reciprocal()).clamp(-FP8_MAX, FP8_MAX)
    if is_root:
        scaled = torch.where(x > 0, scaled.clamp_min(FP8_LEAST), scaled)
    return scaled.to(FP8).reshape(-1), scale.reshape(-1)


def _from8(codes, scale):
    return (codes.float().reshape(-1, BLOCK) * scale[:, None]).reshape(-1)


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    call = case["call"]
    if call in ("sort", "join"):
        pairs, T, D, e = case["tokens"] * case["top_k"], case["tokens"], case["dim"], BYTES[case["dtype"]]
        if call == "sort":  # indices in, pair and row out; rows in and out; with its gradient the same back
            return {"bytes": 12 * pairs + (T + pairs) * D * e * (2 if case["train"] else 1), "flops": pairs * D if case["train"] else 0}
        # rows, output gradient, weights, places in; sum, rows' and weights' gradients out
        return {"bytes": (2 * pairs + 2 * T) * D * e + 12 * pairs, "flops": 5 * pairs * D}
    if call in ("forward", "backward"):
        R, K, I, O, e = case["rows"], case["heads"], case["fan_in"], case["fan_out"], BYTES[case["dtype"]]
        used = min(K, R)  # heads without rows need no weights
        if call == "forward":
            return {"bytes": R * (I + O) * e + used * O * (I * e + 4), "flops": 2 * R * I * O}
        read = R * (I + O * (2 if case["relu"] else 1)) * e + used * O * I * e
        return {"bytes": read + R * I * e + 4 * K * O * (I + 1), "flops": 4 * R * I * O}
    n, e = sum(_sizes(case)), BYTES[case["dtype"]]
    moments = 16 if case["bits"] == 32 else 4 + 16.0 / BLOCK
    return {"bytes": n * (2 * e + BYTES[case["grad"]] + moments + (2 if case["copy"] else 0)), "flops": 15 * n}


# ---- the same in 64 bits --------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    call = case["call"]
    f8 = torch.float64
    if call in ("sort", "join"):
        ids = s["ids"].cpu().numpy().reshape(-1)
        K, k = case["heads"], case["top_k"]
        lists = [np.flatnonzero(ids == h) for h in range(K)]
        counts = [len(p) for p in lists]
        pair = np.concatenate(lists + [np.flatnonzero((ids < 0) | (ids >= K))])
        place = np.argsort(pair)
        offsets = np.concatenate([[0], np.cumsum(counts)])
        has = place < offsets[-1]
        row = np.where(has, place, -1 - place)
        pair_d, place_d, has_d = (torch.from_numpy(v).cuda() for v in (pair, place, has))
        if call == "sort":
            rows = s["x"].to(f8)[pair_d // k]
            rows[int(offsets[-1]):] = 0
            dx = None
            if case["train"]:
                dx = torch.zeros(s["x"].shape, dtype=f8, device="cuda")
                of = pair_d[:int(offsets[-1])] // k
                dx.index_add_(0, of, s["grad"][:int(offsets[-1])].to(f8))
            return {"offsets": offsets.astype(np.int32), "pair": pair.astype(np.int32),
                    "row": row.astype(np.int32).reshape(s["ids"].shape), "rows": rows, "dx": dx}
        weights = torch.where(has_d, s["weights"].reshape(-1).to(f8), 0.0)
        y = torch.zeros(case["tokens"], case["dim"], dtype=f8, device="cuda")
        of = pair_d // k
        y.index_add_(0, of, s["rows"].to(f8) * weights[pair_d][:, None])
        drows = s["grad"].to(f8)[of] * weights[pair_d][:, None]
        dots = (s["grad"].to(f8)[of] * s["rows"].to(f8)).sum(1)
        dweights = torch.where(has_d, dots[place_d], 0.0).reshape(s["ids"].shape)
        return {"y": y, "drows": drows, "dweights": dweights}
    if call in ("forward", "backward"):
        R, K, I, O = (case[n] for n in ("rows", "heads", "fan_in", "fan_out"))
        ends = s["offsets"].tolist()
        if call == "forward":
            y = torch.zeros(R, O, dtype=f8, device="cuda")
            for h in range(K):
                a, b = ends[h], ends[h + 1]
                y[a:b] = torch.addmm(s["b"][h].to(f8), s["x"][a:b].to(f8), s["w"][h].to(f8).T)
            return {"y": y.clamp_min(0) if case["relu"] else y}
        dx = torch.zeros(R, I, dtype=f8, device="cuda")
        dw, db = torch.zeros(K, O, I, dtype=f8, device="cuda"), torch.zeros(K, O, dtype=f8, device="cuda")
        for h in range(K):
            a, b = ends[h], ends[h + 1]
            dz = s["grad"][a:b].to(f8)
            if case["relu"]:
                dz = torch.where(s["y"][a:b] > 0, dz, 0.0)
            dx[a:b], dw[h], db[h] = dz @ s["w"][h].to(f8), dz.T @ s["x"][a:b].to(f8), dz.sum(0)
        return {"dx": dx, "dw": dw, "db": db}
    t = s["step"] + 1
    grad = s["g"].to(f8) * s["scale"].to(f8)
    m, v = s["m"].to(f8), s["v"].to(f8)
    if case["bits"] == 8:
        m = m * s["m_scale"].to(f8).repeat_interleave(BLOCK)
        v = (v * s["v_scale"].to(f8).repeat_interleave(BLOCK)) ** 2
    m, v = BETA1 * m + (1 - BETA1) * grad, BETA2 * v + (1 - BETA2) * grad * grad
    p = s["p"].to(f8) * (1 - LR * DECAY)
    p -= LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    r = {"p": p, "copy": p if case["copy"] else None, "m": m, "v": v, "m_scale": None, "v_scale": None}
    if case["bits"] == 8:  # the codes are the nearest ones of e4m3 to a moment over its block's scale
        for name, x in (("m", m), ("v", torch.sqrt(v))):
            scale = (x.reshape(-1, BLOCK).abs().amax(1) / FP8_MAX).clamp_min(SCALE_LEAST)
            over = x / scale.repeat_interleave(BLOCK)
            step = torch.exp2(torch.floor(torch.log2(over.abs().clamp_min(2.0 ** -6))) - 3)
            code = torch.round(over / step) * step
            if name == "v":
                code = torch.where(x > 0, code.clamp_min(FP8_LEAST), code)
            r[name], r[name + "_scale"] = code, scale
    return r
