"""Further operators that train and serve a mixture of heads, as a program calls them.

A case names one operator and its sizes:

  gated       every head's gated layer on its rows: act(gate) * up, with what its gradients need where a training
              step keeps it
  gated_back  the gradients of that layer: inputs, weights, biases
  lookup      rows of a table picked by the samples' ids and scaled (a code for each image, a feature for each cell);
              with train also the table's gradient, a sum over each row's samples.  A sample may have no row.
  orthogonal  every head's matrix orthogonalised by five steps of a quintic iteration
  muon        one step over the heads' weight tensors: momentum, the orthogonalised direction, decay

Each has a plain form (elementary torch operations in float32) and, where own is true, the calls of
paper_2011_12490_amd.heads.  exact() computes the same in float64.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
ACTS = ["silu", "gelu", "relu", "sigmoid"]
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
STEPS, QUINTIC, NORM_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def listed():
    return [
        # one sample a head through wide heads, as a serving loop has them: the weights are what is read
        _gated("gated_few", "gated", 16, 16, 1024, 4096, "bf16", "silu", False, False),
        # hidden layers of 8x256 heads on a ragged training batch
        _gated("gated_hidden", "gated", 262139, 16, 256, 256, "bf16", "silu", True, True),
        # wide heads at a large batch, not trained
        _gated("gated_wide", "gated", 32768, 8, 2048, 4096, "bf16", "silu", False, False),
        # the first layer of 8x128 heads in float32 (63 inputs), trained
        _gated("gated_first_fp32", "gated", 98301, 16, 63, 128, "fp32", "gelu", True, True),
        # a hidden layer of 8x128 heads, two heads a sample
        _gated("gated_back_hidden", "gated_back", 131072, 16, 128, 128, "bf16", "silu", True, True),
        # wide heads, all gradients
        _gated("gated_back_wide", "gated_back", 16384, 8, 2048, 4096, "bf16", "silu", False, True),
        # a few rays' codes: launches and latency
        _lookup("lookup_few", 64, 500, 48, "bf16", 0.0, False),
        # a training batch of 2,048 rays of 128 samples, each with its image's code of 48 values; many samples a row
        _lookup("lookup_codes", 2048 * 128, 1000, 48, "fp32", 0.03, True),
        # features of many cells; a few samples a row, some rows none
        _lookup("lookup_large", 524288, 200000, 512, "bf16", 0.03, True),
        # odd matrices in float32
        _orthogonal("orthogonal_odd", 24, 300, 701, "fp32"),
        # the hidden layers of 16 heads of 8x128 behind 63 inputs, bf16 copies kept for the matrix units
        _muon("muon_heads", 16, 8, 128, 128, 63, "fp32", "fp32", True),
        # wide heads, there and back, in bf16
        _muon("muon_wide", 8, 2, 2048, 4096, 0, "bf16", "bf16", False),
    ]


def _gated(name, call, rows, heads, fan_in, fan_out, dtype, act, bias, keep, dropped=0.0):
    return _named(name, call=call, rows=rows, heads=heads, fan_in=fan_in, fan_out=fan_out, dtype=dtype, act=act, bias=bias,
                  keep=keep, dropped=dropped)


def _lookup(name, samples, table, dim, dtype, dropped, train):
    return _named(name, call="lookup", samples=samples, table=table, dim=dim, dtype=dtype, dropped=dropped, train=train)


def _orthogonal(name, heads, fan_out, fan_in, dtype):
    return _named(name, call="orthogonal", heads=heads, fan_out=fan_out, fan_in=fan_in, dtype=dtype)


def _muon(name, heads, layers, fan_out, fan_in, first, dtype, grad, copy):
    return _named(name, call="muon", heads=heads, layers=layers, fan_out=fan_out, fan_in=fan_in, first=first, dtype=dtype,
                  grad=grad, copy=copy)


def _named(name, **case):
    return dict(case, name=name) if name else case


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["gated", "gated", "gated_back", "gated_back", "lookup", "lookup", "orthogonal", "muon"])
    while True:
        dtype = rng.choice(["fp32", "bf16"])
        dropped = rng.choice([0.0, 0.0, 0.03, 0.3])
        if call in ("gated", "gated_back"):
            # odd widths are those of encodings and skip inputs
            heads, rows = _spread(rng, 2, 128), _spread(rng, 1, 262144)
            fan_in = rng.choice([27, 39, 63, 64, 91, 128, 155, 256, 283, 319, _spread(rng, 16, 2048), 64 * rng.randint(1, 32)])
            fan_out = rng.choice([3, 32, 64, 64, 128, 128, 256, 256, _spread(rng, 16, 4096), 64 * rng.randint(1, 64)])
            cost = 4.0 * rows * fan_in * fan_out * (2 if call == "gated_back" else 1) * (4 if dtype == "fp32" else 1)
            if cost > 8e11 or rows * (fan_in + 4 * fan_out) > 1 << 28 or heads * fan_in * fan_out > 1 << 26:
                continue
            return _gated(None, call, rows, heads, fan_in, fan_out, dtype, rng.choice(ACTS), rng.random() < 0.6,
                          call == "gated_back" or rng.random() < 0.5, dropped)
        if call == "lookup":
            samples, table, dim = _spread(rng, 1, 1 << 20), _spread(rng, 2, 1 << 20), _spread(rng, 1, 1024)
            if samples * dim > 1 << 27 or table * dim > 1 << 27:
                continue
            return _lookup(None, samples, table, dim, dtype, dropped, rng.random() < 0.7)
        heads, fan_out, fan_in = _spread(rng, 1, 64), _spread(rng, 8, 2048), _spread(rng, 8, 2048)
        layers = rng.randint(1, 8) if call == "muon" else 1
        if _iteration_flops(fan_out, fan_in) * heads * layers > 2e12 or heads * layers * fan_out * fan_in > 1 << 26:
            continue
        if call == "orthogonal":
            return _orthogonal(None, heads, fan_out, fan_in, dtype)
        return _muon(None, heads, layers, fan_out, fan_in, rng.choice([0, 27, 63, fan_in + 63]), dtype, rng.choice(["fp32", dtype]),
                     dtype == "fp32" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------

def _shares(rng, heads):
    """How often each head is taken: far from even, as cells of a scene are."""
    p = rng.gamma(1.5, 1.0, heads) + 0.02
    return p / p.sum()


def _shapes(case):
    """[fan_out, fan_in] of each tensor's matrices: a first layer of its own, layers there and, in pairs, back."""
    O, I = case["fan_out"], case["fan_in"]
    rest = [(O, I) if i % 2 == 0 or O == I else (I, O) for i in range(case["layers"])]
    return ([(O, case["first"])] if case["first"] else []) + rest


def _gradient(rand, heads, fan_out, fan_in):
    """Matrices whose directions differ in size by a few powers of e, as sums over a batch's rows have them."""
    rank = min(fan_out, fan_in)
    size = torch.exp(-4.0 * torch.arange(rank, device="cuda") / rank)
    return rand(heads, fan_out, rank) * size @ rand(heads, rank, fan_in) * (1e-3 / rank ** 0.5)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    call = case["call"]
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    dtype = TYPES[case["dtype"]]
    if call in ("gated", "gated_back"):
        R, K, I, O = (case[n] for n in ("rows", "heads", "fan_in", "fan_out"))
        counts = rng.multinomial(R - int(R * case["dropped"]), _shares(rng, K))
        s = {"case": case, "counts": [int(n) for n in counts],
             "offsets": torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda"),
             "x": rand(R, I).to(dtype), "w": (rand(K, 2, O, I) * I ** -0.5).to(dtype),
             "b": 0.1 * rand(K, 2, O) if case["bias"] else None}
        if call == "gated_back":
            s["grad"] = (0.1 * rand(R, O)).to(dtype)
            s["pre"] = (1.5 * rand(R, 2 * O)).to(dtype)  # gates and ups, as the layer kept them
        return s
    if call == "lookup":
        T, V, D = case["samples"], case["table"], case["dim"]
        # a few rows are met often, many seldom, in no order
        often = torch.randperm(V, generator=g, device="cuda")
        ids = often[(V * torch.rand(T, generator=g, device="cuda").double() ** 2).long().clamp_max(V - 1)]
        if case["dropped"]:
            ids = torch.where(torch.rand(T, generator=g, device="cuda") < case["dropped"], -1, ids)
        return {"case": case, "ids": ids.int(), "table": rand(V, D).to(dtype), "scale": D ** 0.5,
                "grad": (0.1 * rand(T, D)).to(dtype) if case["train"] else None}
    K = case["heads"]
    if call == "orthogonal":
        return {"case": case, "x": _gradient(rand, K, case["fan_out"], case["fan_in"]).to(dtype)}
    shapes = _shapes(case)
    p = [(0.05 * rand(K, o, i)).to(dtype) for o, i in shapes]
    s = {"case": case, "scale": torch.rand(1, generator=g, device="cuda") * 0.5 + 0.5, "p": p,
         "copy": [torch.zeros_like(x, dtype=torch.bfloat16) for x in p] if case["copy"] else None,
         "g": [_gradient(rand, K, o, i).to(TYPES[case["grad"]]) for o, i in shapes],
         "m": [5.0 * _gradient(rand, K, o, i) for o, i in shapes]}
    if own:
        from paper_2011_12490_amd import heads
        s["optimizer"] = heads.Muon(s["p"], s["g"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, copies=s["copy"], m=s["m"])
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s["case"], s)


def _run_own(case, s):
    from paper_2011_12490_amd import heads
    call = case["call"]
    if call == "gated":
        y, pre = heads.gated(s["x"], s["w"], s["b"], s["offsets"], act=case["act"], keep=case["keep"])
        return {"y": y, "pre": pre}
    if call == "gated_back":
        dx, dw, db = heads.gated_backward(s["grad"], s["pre"], s["x"], s["w"], s["offsets"], act=case["act"])
        return {"dx": dx, "dw": dw, "db": db}
    if call == "lookup":
        rows = heads.lookup(s["table"], s["ids"], scale=s["scale"])
        grad = heads.lookup_backward(s["grad"], s["ids"], case["table"], scale=s["scale"]) if case["train"] else None
        return {"rows": rows, "grad": grad}
    if call == "orthogonal":
        return {"x": heads.orthogonalise(s["x"])}
    s["optimizer"].step(grad_scale=s["scale"])
    return {n: s[n] for n in ("p", "copy", "m")}


def _act(g, act):
    """The activation and its derivative."""
    if act == "relu":
        return g.clamp_min(0), (g > 0).to(g.dtype)
    if act == "gelu":
        half = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
        return g * half, half + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    gate = 1 / (1 + torch.exp(-g))
    if act == "sigmoid":
        return gate, gate * (1 - gate)
    return g * gate, gate * (1 + g * (1 - gate))


def _run_plain(case, s):
    call = case["call"]
    if call in ("gated", "gated_back"):
        # a head's rows lie one after another, so each head is one product; the counts are known on the host here
        K, I, O, dtype = case["heads"], case["fan_in"], case["fan_out"], s["x"].dtype
        x, w = s["x"].float(), s["w"].float().reshape(K, 2 * O, I)
        headed, rest = sum(s["counts"]), x.shape[0] - sum(s["counts"])
        xs = torch.split(x[:headed], s["counts"])
        if call == "gated":
            pre = torch.cat([p @ w[h].T for h, p in enumerate(xs)] + [x.new_zeros(rest, 2 * O)])
            if s["b"] is not None:
                of = torch.repeat_interleave(torch.arange(K, device="cuda"), s["offsets"].diff(), output_size=headed)
                pre[:headed] += s["b"].reshape(K, 2 * O)[of]
            y = _act(pre[:, :O], case["act"])[0] * pre[:, O:]
            y[headed:] = 0
            return {"y": y.to(dtype), "pre": pre.to(dtype) if case["keep"] else None}
        dy, up = s["grad"].float(), s["pre"][:, O:].float()
        value, slope = _act(s["pre"][:, :O].float(), case["act"])
        dz = torch.split(torch.cat([dy * up * slope, dy * value], dim=1)[:headed], s["counts"])
        dx = torch.cat([z @ w[h] for h, z in enumerate(dz)] + [x.new_zeros(rest, I)])
        dw = torch.stack([z.T @ p for z, p in zip(dz, xs)]).reshape(K, 2, O, I)
        db = torch.stack([z.sum(0) for z in dz]).reshape(K, 2, O)
        return {"dx": dx.to(dtype), "dw": dw.to(dtype), "db": db}
    if call == "lookup":
        ids, has, scale = s["ids"].long(), (s["ids"] >= 0)[:, None], s["scale"]
        rows = (torch.where(has, s["table"][ids.clamp_min(0)].float(), 0.0) * scale).to(s["table"].dtype)
        grad = None
        if case["train"]:
            grad = torch.zeros(case["table"] + 1, case["dim"], device="cuda")  # the last row: samples without one
            grad = grad.index_add_(0, torch.where(s["ids"] < 0, case["table"], ids), s["grad"].float())[:-1] * scale
        return {"rows": rows, "grad": grad}
    if call == "orthogonal":
        return {"x": _orthogonalised(s["x"].float()).to(s["x"].dtype)}
    copies = s["copy"] or [None] * len(s["p"])
    for p, grad, m, copy in zip(s["p"], s["g"], s["m"], copies):
        scaled = grad.float() * s["scale"]
        m.mul_(MOMENTUM).add_(scaled)
        new = p.float() * (1 - LR * DECAY) - _orthogonalised(scaled + m * MOMENTUM) * (LR * _size(p))
        p.copy_(new)
        if copy is not None:
            copy.copy_(new)
    return {n: s[n] for n in ("p", "copy", "m")}


def _size(p):
    """How large a tensor's steps are: tall matrices have longer rows of small values."""
    return max(1.0, p.shape[-2] / p.shape[-1]) ** 0.5


def _orthogonalised(x):
    a, b, c = QUINTIC
    x = (x.double() / (x.double().square().sum((-2, -1), keepdim=True).sqrt() + NORM_EPS)).float()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT.contiguous() if tall else x
    for _ in range(STEPS):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT.contiguous() if tall else x


# ---- what a pass cannot do without ----------------------------------------------

def _iteration_flops(fan_out, fan_in):
    """Of the five steps on one matrix: x x^T and its square are symmetric, and half of each is enough."""
    m, n = min(fan_out, fan_in), max(fan_out, fan_in)
    return STEPS * (m * m * n + m ** 3 + 2 * m * m * n)


def work(case):
    call, e = case["call"], BYTES[case["dtype"]]
    if call in ("gated", "gated_back"):
        R, K, I, O = case["rows"], case["heads"], case["fan_in"], case["fan_out"]
        used = min(K, R)  # heads without rows need no weights
        if call == "gated":
            return {"bytes": R * (I + (3 if case["keep"] else 1) * O) * e + used * 2 * O * (I * e + (4 if case["bias"] else 0)),
                    "flops": 4 * R * I * O}
        return {"bytes": R * (2 * I + 3 * O) * e + (used + K) * 2 * O * I * e + 8 * K * O, "flops": 8 * R * I * O}
    if call == "lookup":
        T, V, D = case["samples"], case["table"], case["dim"]
        met = V * (1 - math.exp(-T / V))  # about as many rows as samples reach
        forward = 4 * T + (min(met, T) + T) * D * e
        return {"bytes": forward + (T * D * e + 4 * V * D if case["train"] else 0), "flops": (2 if case["train"] else 1) * T * D}
    if call == "orthogonal":
        n = case["heads"] * case["fan_out"] * case["fan_in"]
        return {"bytes": 2 * n * e, "flops": case["heads"] * _iteration_flops(case["fan_out"], case["fan_in"])}
    shapes = _shapes(case)
    n = case["heads"] * sum(o * i for o, i in shapes)
    return {"bytes": n * (2 * e + BYTES[case["grad"]] + 8 + (2 if case["copy"] else 0)),
            "flops": case["heads"] * sum(_iteration_flops(o, i) for o, i in shapes)}


# ---- the same in 64 bits --------------------------------------------------------

def _exact_act(act):
    if act == "relu":
        return lambda v: torch.where(v > 0, v, torch.zeros_like(v)), lambda v: torch.where(v > 0, 1.0, 0.0).to(v.dtype)
    if act == "sigmoid":
        return torch.sigmoid, lambda v: torch.sigmoid(v) * torch.sigmoid(-v)
    if act == "silu":
        return lambda v: v * torch.sigmoid(v), lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)
    below = lambda v: torch.erfc(-v / math.sqrt(2.0)) / 2  # noqa: E731
    return lambda v: v * below(v), lambda v: below(v) + v * torch.exp(-v * v / 2) / math.sqrt(2.0 * math.pi)


def _exact_direction(x):
    """The iteration on singular values: x's left and right directions stay, each value v becomes a v + b v^3 + c v^5."""
    a, b, c = QUINTIC
    x = x / (torch.linalg.vector_norm(x) + NORM_EPS)
    wide = x if x.shape[0] <= x.shape[1] else x.T
    eye = torch.eye(wide.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        s = torch.mm(wide, wide.T)
        wide = torch.mm(torch.addmm(a * eye, s, b * eye + c * s), wide)
    return wide if x.shape[0] <= x.shape[1] else wide.T


def exact(case, seed):
    s = prepare(case, seed)
    call, f8 = case["call"], torch.float64
    if call in ("gated", "gated_back"):
        R, K, I, O = (case[n] for n in ("rows", "heads", "fan_in", "fan_out"))
        ends = s["offsets"].tolist()
        f, df = _exact_act(case["act"])
        new = lambda *shape: torch.zeros(*shape, dtype=f8, device="cuda")  # noqa: E731
        if call == "gated":
            y, pre = new(R, O), new(R, 2, O)
            for h, (start, end) in enumerate(zip(ends, ends[1:])):
                x = s["x"][start:end].to(f8)
                for part in range(2):
                    pre[start:end, part] = x @ s["w"][h, part].to(f8).T
                    if s["b"] is not None:
                        pre[start:end, part] += s["b"][h, part].to(f8)
                y[start:end] = f(pre[start:end, 0]) * pre[start:end, 1]
            return {"y": y, "pre": pre.reshape(R, 2 * O) if case["keep"] else None}
        dx, dw, db = new(R, I), new(K, 2, O, I), new(K, 2, O)
        for h, (start, end) in enumerate(zip(ends, ends[1:])):
            x, dy = s["x"][start:end].to(f8), s["grad"][start:end].to(f8)
            gate, up = s["pre"][start:end].to(f8).chunk(2, dim=1)
            for part, dz in enumerate((dy * up * df(gate), dy * f(gate))):
                dx[start:end] += dz @ s["w"][h, part].to(f8)
                dw[h, part], db[h, part] = dz.T @ x, dz.sum(0)
        return {"dx": dx, "dw": dw, "db": db}
    if call == "lookup":
        has = s["ids"] >= 0
        rows = torch.zeros(case["samples"], case["dim"], dtype=f8, device="cuda")
        rows[has] = s["table"].to(f8)[s["ids"][has].long()] * s["scale"]
        grad = None
        if case["train"]:
            grad = torch.zeros(case["table"], case["dim"], dtype=f8, device="cuda")
            grad.index_add_(0, s["ids"][has].long(), s["grad"][has].to(f8) * s["scale"])
        return {"rows": rows, "grad": grad}
    if call == "orthogonal":
        return {"x": torch.stack([_exact_direction(x.to(f8)) for x in s["x"]])}
    p, moments = [], []
    for w, grad, m in zip(s["p"], s["g"], s["m"]):
        grad = grad.to(f8) * s["scale"].to(f8)
        m = MOMENTUM * m.to(f8) + grad
        way = torch.stack([_exact_direction(x) for x in grad + MOMENTUM * m])
        moments.append(m)
        p.append(w.to(f8) - LR * (DECAY * w.to(f8) + math.sqrt(max(1.0, w.shape[1] / w.shape[2])) * way))
    return {"p": p, "copy": p if case["copy"] else None, "m": moments}
