"""Operators right before an answer is drawn and right before parameters are stepped: timing cases.

  adjust       qsv_adjust: penalties for repeated outcomes, biases and masks on rows of scores
  adjust_grad  qsv_adjust_grad: its backward pass, with the gradients of a bias that all rows share and of the rows' own
  clip         qsv_clip_grads: the norm of many tensors' gradients together, and the gradients scaled to a highest norm
  adam         qsv_adam_clipped: Adam's step over many tensors, with that scaling on the way

``run`` computes an operator in its plain form, or (``own``) by the library's calls.
"""
import math

import torch

own = False

FLOATS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}

# Tensors of a model: rows x columns (+ columns of padding behind a row), or the length of a vector.
SETS = {
    # the angles of an encoder and a decoder, a read-out's weights and bias
    "circuit": "320 320 10x64 10",
    # some dozen small layers, odd sizes among them
    "layers": " ".join(["64x64 64 64x257 257 33x65 1 127x129 999"] * 6),
    # gradients of scores with padded rows, and of biases
    "scores": "4096x32768+8 32768 513x50021+3 7",
    # more than a hundred matrices
    "stack": " ".join(["768x768 768 768x2048 2048"] * 48),
}


def _shapes(text):
    """(rows, columns, columns of padding) of each tensor."""
    got = []
    for t in text.split():
        t, _, pad = t.partition("+")
        rows, _, cols = t.rpartition("x")
        got.append((int(rows or 1), int(cols), int(pad or 0)))
    return got


def _adjust(name, src, rows, cols, prior=0, penalties=0, bias=0, entries=0, masks=0, allowed=1.0, pad=0, in_place=0):
    c = dict(op="adjust", src=src, rows=rows, cols=cols, prior=prior, penalties=penalties, bias=bias, entries=entries, masks=masks,
             allowed=allowed, pad=pad, in_place=in_place)
    return dict(c, name=name) if name else c


def _adjust_grad(name, *a, **k):
    return dict(_adjust(name, *a, **k), op="adjust_grad")


def _tensors(name, op, src, tensors, norm, t=1):
    """norm: the highest one; 0: it is worked out alone."""
    c = dict(op=op, src=src, tensors=tensors, norm=norm)
    if op == "adam":
        c["t"] = t
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sequence that is decoded: penalties over what it has so far, all latency
        _adjust("adjust_bf16_1x32768", "bf16", 1, 32768, prior=700, penalties=1),
        # a few sequences with everything: own penalties, own biases, grammars of which one leaves nothing, an odd vocabulary
        _adjust("adjust_f16_24x50021", "f16", 24, 50021, prior=2000, penalties=1, bias=1, entries=40, masks=5, allowed=0.4, pad=3),
        # a serving batch under grammars alone, over the scores themselves
        _adjust("adjust_f32_256x131072_masks", "f32", 256, 131072, masks=64, allowed=0.05, in_place=1),
        # a large serving batch: penalties, a shared bias and grammars
        _adjust("adjust_bf16_512x131072", "bf16", 512, 131072, prior=1024, penalties=1, bias=1, masks=32, allowed=0.5),
        # long contexts of a few sequences
        _adjust("adjust_f16_8x200003_long", "f16", 8, 200003, prior=32768, penalties=1, entries=300, pad=1),
        # the backward pass of a small step with everything
        _adjust_grad("adjust_grad_f32_16x1000", "f32", 16, 1000, prior=100, penalties=1, bias=1, entries=8, masks=3, allowed=0.5),
        # a training step under grammars with a learned bias
        _adjust_grad("adjust_grad_bf16_4096x32768", "bf16", 4096, 32768, bias=1, masks=256, allowed=0.3),
        # an odd number of rows, an odd vocabulary, histories
        _adjust_grad("adjust_grad_f16_513x50021", "f16", 513, 50021, prior=256, penalties=1, bias=1, entries=20, masks=7, allowed=0.9, pad=3),
        # gradients of a circuit and its read-out: all latency
        _tensors("clip_f32_circuit", "clip", "f32", SETS["circuit"], 0.5),
        # large gradients of scores, padded rows, more than the memory-side cache holds
        _tensors("clip_bf16_scores", "clip", "bf16", SETS["scores"], 0.25),
        # a step over some dozen small layers
        _tensors("adam_f32_layers", "adam", "f32", SETS["layers"], 1.0, t=3),
        # a large step with gradients of 16 bits
        _tensors("adam_bf16_stack", "adam", "bf16", SETS["stack"], 1.0, t=1000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case; sizes stay below the largest listed ones of their operator."""
    op = rng.choice(["adjust", "adjust", "adjust_grad", "clip", "adam"])
    if op in ("adjust", "adjust_grad"):
        cols = _log_int(rng, 16, 262144)
        rows = _log_int(rng, 1, max(1, min(4096, (1 << 25) // cols)))
        prior = rng.choice([0, 1]) * _log_int(rng, 1, max(1, min(32768, (1 << 21) // rows)))
        masks = rng.choice([0, 1]) * _log_int(rng, 1, 64)
        penalties, entries = int(prior > 0), rng.choice([0, 0, 1]) * _log_int(rng, 1, min(300, cols))
        bias = rng.randint(0, 1)
        what = dict(prior=prior, penalties=penalties, bias=bias, entries=entries, masks=masks,
                    allowed=rng.choice([0.01, 0.3, 0.7, 0.99]) if masks else 1.0, pad=rng.choice([0, 0, 1, 8]))
        src = rng.choice(["f32", "f16", "bf16"])
        if op == "adjust":
            return _adjust("", src, rows, cols, **what)
        return _adjust_grad("", src, rows, cols, **what)
    count = _log_int(rng, 1, 200)
    room = _log_int(rng, 100, 1 << 25)
    tensors = []
    for _ in range(count):
        n = _log_int(rng, 1, max(2, 2 * room // count))
        rows = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, min(4096, n)))
        pad = rng.choice([0, 0, 0, 1, 8]) if op == "clip" else 0
        tensors.append("%dx%d+%d" % (rows, max(1, n // rows), pad))
    norm = rng.choice([0.1, 1.0, 1.0, 1e6]) if op == "adam" else rng.choice([0.1, 1.0, 1e6, 0.0])
    return _tensors("", op, rng.choice(["f32", "f16", "bf16"]), " ".join(tensors), norm, t=_log_int(rng, 1, 10000))


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _int(g, low, high, *shape):
    return torch.randint(low, high, shape, generator=g, device="cuda", dtype=torch.int32)


def _rows_of(g, rows, choices):
    """One of `choices` for each row."""
    return torch.tensor(choices, dtype=torch.float32, device="cuda")[_int(g, 0, len(choices), rows).long()]


def _masks(c, g):
    """Bit k % 32 of word k / 32 allows outcome k; of three masks and more the last allows none."""
    words = (c["cols"] + 31) // 32
    got = torch.zeros((c["masks"], words), dtype=torch.int32, device="cuda")
    bit = torch.arange(32, device="cuda", dtype=torch.int64)
    for i in range(c["masks"] if c["masks"] < 3 else c["masks"] - 1):
        on = (_rand(g, words, 32) < c["allowed"]).long() << bit
        got[i] = on.sum(dim=1).to(torch.int32)
    return got


def _prepare_adjust(c, g):
    rows, cols, dtype = c["rows"], c["cols"], FLOATS[c["src"]]
    z = torch.randn((rows, cols + c["pad"]), generator=g, device="cuda")
    z *= _rand(g, rows, 1) * 3.0 + 1.5
    if cols > 64:
        z[:, cols - 5:cols] = -math.inf     # a vocabulary rounded up: columns that stand for nothing
    s = dict(case=c, scores=z.to(dtype)[:, :cols])
    del z
    more = s["more"] = {}
    if c["prior"]:
        n = c["prior"]
        more["prior"] = (_rand(g, rows, n).pow_(3) * cols).to(torch.int32).clamp_(max=cols - 1)    # some outcomes far oftener than others
        more["prior_len"] = _int(g, (n + 1) // 2, n + 1, rows)
        more["prompt_len"] = (_rand(g, rows) * more["prior_len"]).to(torch.int32)
        more["prior"][torch.arange(n, device="cuda").view(1, -1) >= more["prior_len"].view(-1, 1)] = -1
    if c["penalties"]:
        more["repetition"] = _rows_of(g, rows, [1.0, 1.05, 1.1, 1.3])
        if c["op"] == "adjust":
            more["frequency"] = _rows_of(g, rows, [0.0, 0.1, 0.5, -0.2])
            more["presence"] = _rows_of(g, rows, [0.0, 0.3, 1.0])
    if c["bias"] and c["op"] == "adjust":
        more["bias"] = torch.randn((cols,), generator=g, device="cuda") * 0.3
    if c["entries"]:
        more["entry_idx"] = _int(g, 0, cols, rows, c["entries"])
        more["entry_idx"][1::3, c["entries"] - c["entries"] // 3:] = -1       # requests with fewer entries
        if c["op"] == "adjust":
            more["entry_bias"] = torch.randn((rows, c["entries"]), generator=g, device="cuda") * 4.0
    if c["masks"]:
        more["masks"] = _masks(c, g)
        more["mask_of"] = _int(g, 0, c["masks"], rows)
        more["mask_of"][2::7] = -1                                            # requests without a grammar
    like = lambda: torch.zeros((rows, cols + c["pad"]), dtype=dtype, device="cuda")[:, :cols]  # noqa: E731
    if c["op"] == "adjust":
        s["out"] = s["scores"] if c["in_place"] else like()
        return s
    s["grad_out"] = (torch.randn((rows, cols + c["pad"]), generator=g, device="cuda") / rows).to(dtype)[:, :cols]
    s["grad"] = like()
    if c["bias"]:
        s["grad_bias"] = torch.zeros((cols,), device="cuda")
    if c["entries"]:
        s["grad_entry"] = torch.zeros((rows, c["entries"]), device="cuda")
    return s


def _views(flat, shapes):
    """The tensors that lie one behind the other in a program's one buffer."""
    got, at = [], 0
    for rows, cols, pad in shapes:
        n = rows * (cols + pad)
        got.append(flat[at:at + n].view(rows, cols + pad)[:, :cols])
        at += n
    return got


def _prepare_tensors(c, g):
    """Gradients are tensors of their own; what the call writes lies in one buffer each, as programs keep parameters and moments."""
    shapes, dtype = _shapes(c["tensors"]), FLOATS[c["src"]]
    s = dict(case=c, grads=[], norm=torch.zeros((1,), device="cuda"))
    total = sum(rows * (cols + pad) for rows, cols, pad in shapes)
    scales = [0.02 * 2.0 ** (i % 5 - 3) for i in range(len(shapes))]         # layers whose gradients differ in size
    for (rows, cols, pad), scale in zip(shapes, scales):
        s["grads"].append(torch.randn((rows, cols + pad), generator=g, device="cuda").mul_(scale).to(dtype)[:, :cols])
    if c["op"] == "clip":
        s["out"] = torch.zeros((total,), dtype=dtype, device="cuda")
        return s
    s["params"] = torch.randn((total,), generator=g, device="cuda").mul_(0.05)
    s["m"] = torch.randn((total,), generator=g, device="cuda")
    s["v"] = torch.rand((total,), generator=g, device="cuda").add_(0.5)
    for m, v, scale in zip(_views(s["m"], shapes), _views(s["v"], shapes), scales):
        m.mul_(scale * 0.3)
        v.mul_(scale * scale)
    return s


def _handle(s):
    """A context of the library and the lists of tensors, as a program keeps them."""
    from paper_2602_13140_amd import binding as qb
    c, need = s["case"], qb.qsv_workspace_bytes(1, 1)
    if c["op"] == "adjust_grad":
        need = max(need, qb.qsv_adjust_grad_workspace_bytes(c["rows"], c["cols"]))
    s["ctx"] = qb.Context(1, 1, ws_bytes=need)
    if c["op"] == "clip":
        s["list"] = qb.TensorList(s["grads"])
        s["out_list"] = qb.TensorList(_views(s["out"], _shapes(c["tensors"])))
    if c["op"] == "adam":
        s["list"] = qb.AdamList(*(s[k] if k == "grads" else _views(s[k], _shapes(c["tensors"])) for k in ("params", "grads", "m", "v")))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(7919 * int(seed) + 101)
    s = _prepare_adjust(case, g) if case["op"] in ("adjust", "adjust_grad") else _prepare_tensors(case, g)
    if own:
        _handle(s)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _history(more, rows, cols):
    """Which outcomes a row has had, and how often behind its prompt."""
    at, place = more["prior"].long(), torch.arange(more["prior"].shape[1], device="cuda").view(1, -1)
    real = (at >= 0) & (at < cols) & (place < more["prior_len"].view(-1, 1))
    later = real & (place >= more["prompt_len"].view(-1, 1))
    at = torch.where(real, at, cols)
    seen = torch.zeros((rows, cols + 1), dtype=torch.bool, device="cuda").scatter_(1, at, True)
    count = torch.zeros((rows, cols + 1), dtype=torch.int32, device="cuda").scatter_add_(1, at, later.to(torch.int32))
    return seen[:, :cols], count[:, :cols].float()


def _allowed(more, cols):
    of = more["mask_of"].long()
    bits = more["masks"][of.clamp(min=0)].unsqueeze(2) >> torch.arange(32, device="cuda", dtype=torch.int32)
    return ((bits & 1) == 1).flatten(1)[:, :cols] | (of < 0).view(-1, 1)


def _plain_adjust(s):
    c, more = s["case"], s["more"]
    rows, cols = c["rows"], c["cols"]
    v = s["scores"].float()
    if c["prior"]:
        seen, count = _history(more, rows, cols)
        by = more["repetition"].view(-1, 1)
        v = torch.where(seen, torch.where(v > 0, v / by, v * by), v)
        v = v - more["frequency"].view(-1, 1) * count - more["presence"].view(-1, 1) * (count > 0)
    if c["bias"]:
        v = v + more["bias"]
    if c["entries"]:
        at = more["entry_idx"].long()
        real = (at >= 0) & (at < cols)
        own_bias = torch.zeros_like(v).scatter_add_(1, torch.where(real, at, 0), torch.where(real, more["entry_bias"], 0.0))
        v = v + own_bias
    if c["masks"]:
        v = torch.where(_allowed(more, cols), v, -math.inf)
    s["out"].copy_(v)
    return {"out": s["out"]}


def _plain_adjust_grad(s):
    c, more = s["case"], s["more"]
    rows, cols = c["rows"], c["cols"]
    g = s["grad_out"].float()
    if c["masks"]:
        g = torch.where(_allowed(more, cols), g, 0.0)
    got = {}
    if c["bias"]:
        got["grad_bias"] = g.sum(dim=0, dtype=torch.float64).float()
    if c["entries"]:
        at = more["entry_idx"].long()
        real = (at >= 0) & (at < cols)
        got["grad_entry"] = torch.where(real, torch.gather(g, 1, torch.where(real, at, 0)), 0.0)
    if c["prior"]:
        seen, _ = _history(more, rows, cols)
        by = more["repetition"].view(-1, 1)
        g = torch.where(seen, torch.where(s["scores"].float() > 0, g / by, g * by), g)
    got["grad"] = g.to(s["grad_out"].dtype)
    return got


def _norm_and_factor(s):
    """Of sums of squares in 64 bits."""
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        total = total + g.double().square().sum()
    norm = total.sqrt()
    most = s["case"]["norm"] or math.inf
    return norm, torch.where(norm > most, most / norm, 1.0).float()


def _plain_clip(s):
    norm, factor = _norm_and_factor(s)
    got = {"norm": norm.float().view(1)}
    if s["case"]["norm"]:
        for out, g in zip(_views(s["out"], _shapes(s["case"]["tensors"])), s["grads"]):
            out.copy_(g.float() * factor)
        got["out"] = s["out"]
    return got


RATE, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8


def _plain_adam(s):
    norm, factor = _norm_and_factor(s)
    t = s["case"]["t"]
    shapes = _shapes(s["case"]["tensors"])
    for p, g, m, v in zip(_views(s["params"], shapes), s["grads"], _views(s["m"], shapes), _views(s["v"], shapes)):
        g = g.float() * factor
        m.mul_(BETA1).add_(g, alpha=1.0 - BETA1)
        v.mul_(BETA2).add_(g * g, alpha=1.0 - BETA2)
        p.sub_(RATE * (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS))
    return {"norm": norm.float().view(1), "params": s["params"], "m": s["m"], "v": s["v"]}


# ---- one pass --------------------------------------------------------------------------------------------------------
def _kind(s):
    from paper_2602_13140_amd import binding as qb
    return {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16}[s["case"]["src"]]


def _own_adjust(s):
    s["ctx"].qsv_adjust(_kind(s), s["scores"], out=s["out"], **s["more"])
    return {"out": s["out"]}


def _own_adjust_grad(s):
    s["ctx"].qsv_adjust_grad(_kind(s), s["grad_out"], grad=s["grad"], scores=s["scores"], grad_bias=s.get("grad_bias"),
                             grad_entry=s.get("grad_entry"), **s["more"])
    return {k: s[k] for k in ("grad_bias", "grad_entry", "grad") if k in s}


def _own_clip(s):
    most = s["case"]["norm"]
    s["ctx"].qsv_clip_grads(s["list"], most or math.inf, norm=s["norm"], out=s["out_list"] if most else None)
    return {"norm": s["norm"], "out": s["out"]} if most else {"norm": s["norm"]}


def _own_adam(s):
    s["ctx"].qsv_adam_clipped(s["list"], s["case"]["t"], RATE, s["case"]["norm"], BETA1, BETA2, EPS, norm=s["norm"])
    return {k: s[k] for k in ("norm", "params", "m", "v")}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"adjust": _own_adjust, "adjust_grad": _own_adjust_grad, "clip": _own_clip, "adam": _own_adam}[op](s)
    return {"adjust": _plain_adjust, "adjust_grad": _plain_adjust_grad, "clip": _plain_clip, "adam": _plain_adam}[op](s)


def work(case):
    """Scores or gradients read once, results written once (masks over the scores themselves: what they exclude is written).
    A sum for each score that has a bias, ten operations for each earlier outcome and entry; two or three operations for each
    gradient, twenty for a step."""
    c = case
    if c["op"] in ("clip", "adam"):
        n, size = sum(rows * cols for rows, cols, _ in _shapes(c["tensors"])), BYTES[c["src"]]
        if c["op"] == "adam":
            return {"bytes": n * (24 + size) + 4, "flops": 22 * n}
        writes = size if c["norm"] else 0
        return {"bytes": n * (size + writes) + 4, "flops": (3 if writes else 2) * n}
    rows, cols, size = c["rows"], c["cols"], BYTES[c["src"]]
    n = rows * cols
    small = rows * (4 * c["prior"] + 8 * c["entries"] + 24) + c["masks"] * ((cols + 31) // 32) * 4 + (4 * cols if c["bias"] else 0)
    flops = n * (1 if c["bias"] else 0) + 10 * rows * (c["prior"] + c["entries"])
    if c["in_place"]:
        return {"bytes": int(n * (1.0 - c["allowed"]) * 6 / 7) * size + small, "flops": flops}
    return {"bytes": 2 * n * size + small, "flops": flops}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------
def _in_range(v, dtype):
    """Values that the type rounds to infinity."""
    info = torch.finfo(dtype)
    border = info.max * (1.0 + info.eps / 4)
    return torch.where(v.abs() >= border, torch.sign(v) * math.inf, v)


def _row_facts(s, r):
    """Row r: what its history multiplies (0 or 1), the counts, the mask (1: allowed)."""
    c, more = s["case"], s["more"]
    cols = c["cols"]
    seen = count = torch.zeros((cols,), dtype=torch.float64, device="cuda")
    if c["prior"]:
        length, prompt = int(more["prior_len"][r]), int(more["prompt_len"][r])
        had = more["prior"][r, :length].long()
        seen = (torch.bincount(had, minlength=cols) > 0).double()
        count = torch.bincount(had[prompt:], minlength=cols).double()
    allowed = torch.ones((cols,), dtype=torch.bool, device="cuda")
    if c["masks"] and int(more["mask_of"][r]) >= 0:
        words = more["masks"][int(more["mask_of"][r])].long() & 0xffffffff
        k = torch.arange(cols, device="cuda")
        allowed = (words[k // 32] // (2 ** (k % 32))) % 2 == 1
    return seen, count, allowed


def _entries_of(s, r):
    at = s["more"]["entry_idx"][r].long()
    real = (at >= 0) & (at < s["case"]["cols"])
    return at, real


def _exact_adjust(s):
    c, more = s["case"], s["more"]
    out = torch.zeros((c["rows"], c["cols"]), dtype=torch.float64, device="cuda")
    for r in range(c["rows"]):
        seen, count, allowed = _row_facts(s, r)
        z = s["scores"][r].double()
        if c["prior"]:
            by, f, a = (float(more[k][r]) for k in ("repetition", "frequency", "presence"))
            z[seen > 0] = torch.where(z > 0, z / by, z * by)[seen > 0]
            z = z - f * count - a * (count > 0)
        if c["bias"]:
            z = z + more["bias"].double()
        if c["entries"]:
            at, real = _entries_of(s, r)
            z.index_put_((at[real],), more["entry_bias"][r][real].double(), accumulate=True)
        z[~allowed] = -math.inf
        out[r] = _in_range(z, s["scores"].dtype)
    return {"out": out}


def _exact_adjust_grad(s):
    c, more = s["case"], s["more"]
    rows, cols = c["rows"], c["cols"]
    grad = torch.zeros((rows, cols), dtype=torch.float64, device="cuda")
    column = torch.zeros((cols,), dtype=torch.float64, device="cuda")
    entry = torch.zeros((rows, max(1, c["entries"])), dtype=torch.float64, device="cuda")
    for r in range(rows):
        seen, _, allowed = _row_facts(s, r)
        g = s["grad_out"][r].double() * allowed
        column += g
        if c["entries"]:
            at, real = _entries_of(s, r)
            entry[r][real] = g[at[real]]
        if c["prior"]:
            by = float(more["repetition"][r])
            one = torch.ones_like(g)
            slope = torch.where(s["scores"][r] > 0, one / by, one * by)
            g = g * torch.where(seen > 0, slope, one)
        grad[r] = g
    got = {}
    if c["bias"]:
        got["grad_bias"] = column
    if c["entries"]:
        got["grad_entry"] = entry
    got["grad"] = grad
    return got


def _exact_tensors(s):
    c = s["case"]
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
    factor = c["norm"] / norm if 0 < c["norm"] < norm else 1.0
    got = {"norm": torch.tensor([norm], dtype=torch.float64)}
    if c["op"] == "clip":
        if c["norm"]:
            got["out"] = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
            at = 0
            for g, (rows, cols, pad) in zip(s["grads"], _shapes(c["tensors"])):
                for r in range(rows) if pad else [slice(None)]:
                    n = g[r].numel()
                    got["out"][at:at + n] = (g[r].double() * factor).flatten()
                    at += n + pad
        return got
    t = c["t"]
    g = torch.cat([g.double().flatten() for g in s["grads"]]) * factor
    got["m"] = BETA1 * s["m"].double() + (1 - BETA1) * g
    got["v"] = BETA2 * s["v"].double() + (1 - BETA2) * g ** 2
    got["params"] = s["params"].double() - RATE * (got["m"] / (1 - BETA1 ** t)) / (torch.sqrt(got["v"] / (1 - BETA2 ** t)) + EPS)
    return got


def exact(case, seed):
    global own
    was, own = own, False        # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"adjust": _exact_adjust, "adjust_grad": _exact_adjust_grad, "clip": _exact_tensors, "adam": _exact_tensors}[case["op"]](s)
