"""Operators between a model's scores and its answers or its loss: timing cases.

  sample   qsv_sample: outcomes drawn from given uniforms after temperature, min-p, top-k and top-p, from
           scores (log-weights), from probabilities or from the state of a circuit
  distill  qsv_distill: loss against a teacher known by its top logits, and its gradient

``run`` computes an operator in its plain form, or (``own``) by the library's calls.
"""
import math

import numpy as np
import torch

own = False

FLOATS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "probs": 4, "state": 8}


def _sample(name, src, rows, cols, shots, filters, masked=0, pad=0):
    c = dict(op="sample", src=src, rows=rows, cols=cols, shots=shots, filters=filters, masked=masked, pad=pad)
    return dict(c, name=name) if name else c


def _distill(name, src, rows, cols, top, what, temperature=1.0, lse=0, pad=0):
    c = dict(op="distill", src=src, rows=rows, cols=cols, top=top, what=what, temperature=temperature, lse=lse, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sequence that is decoded: one token, all latency
        _sample("sample_bf16_1x32768", "bf16", 1, 32768, 1, "usual"),
        # a few sequences with an own set of filters each, grammar masks, a row with nothing left, an odd vocabulary
        _sample("sample_f16_24x50021", "f16", 24, 50021, 1, "each", masked=1, pad=3),
        # a large serving batch with wide nuclei, several candidates a row
        _sample("sample_f32_256x131072", "f32", 256, 131072, 4, "top_p"),
        # answers read off some qubits of a batch of circuits: their marginal as QSV_M_MARGINAL writes it
        _sample("sample_probs_64x1024", "probs", 64, 1024, 256, "each"),
        # shots of a batch of small circuits at another temperature
        _sample("sample_state_1024x10q", "state", 1024, 1 << 10, 16, "temperature"),
        # shots of one large state without its improbable outcomes
        _sample("sample_state_1x24q", "state", 1, 1 << 24, 4096, "top_p"),
        # a fine-tuning step on labels (one entry a row): the smallest loss with its gradient
        _distill("distill_f32_16x1000", "f32", 16, 1000, 1, "both"),
        # a training step on some thousand positions, softened by a temperature
        _distill("distill_bf16_4096x32768", "bf16", 4096, 32768, 64, "both", temperature=2.0),
        # evaluation: losses alone, an odd vocabulary and an odd number of rows
        _distill("distill_f16_513x50021_loss", "f16", 513, 50021, 20, "loss", lse=1, pad=3),
        # the backward pass by itself, from what the forward pass kept
        _distill("distill_f32_1024x131072_grad", "f32", 1024, 131072, 128, "grad"),
        # a training step of a few long rows
        _distill("distill_bf16_8x131072", "bf16", 8, 131072, 128, "both", lse=1),
        # the largest step
        _distill("distill_bf16_4096x131072", "bf16", 4096, 131072, 128, "both"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case; `room` bounds rows * cols below the largest listed one."""
    if rng.random() < 0.5:
        src = rng.choice(["f32", "f16", "bf16", "probs", "state"])
        cols = 1 << rng.randint(4, 22) if src == "state" else _log_int(rng, 16, 262144)
        rows = _log_int(rng, 1, max(1, min(1024, (1 << 24) // cols)))
        shots = _log_int(rng, 1, 64 if rows > 64 else 1024)
        return _sample("", src, rows, cols, shots, rng.choice(["none", "usual", "top_p", "temperature", "each"]),
                       masked=rng.randint(0, 1), pad=rng.choice([0, 0, 1, 8]) if src in FLOATS else 0)
    cols = _log_int(rng, 50, 131072)
    rows = _log_int(rng, 1, max(1, min(4096, (1 << 27) // cols)))
    return _distill("", rng.choice(["f32", "f16", "bf16"]), rows, cols, _log_int(rng, 1, min(256, cols // 2)),
                    rng.choice(["both", "both", "loss", "grad"]), rng.choice([1.0, 1.0, 2.0, 0.7]), rng.randint(0, 1),
                    rng.choice([0, 0, 1, 8]))


def _scores(c, g):
    """[rows][cols] with a row stride of cols + pad: rows of differing sharpness, as of models more or less sure."""
    rows, cols = c["rows"], c["cols"]
    z = torch.randn((rows, cols + c["pad"]), generator=g, device="cuda")
    z *= torch.rand((rows, 1), generator=g, device="cuda") * 3.0 + 1.5
    return z


def _rows_of(c, g, choices):
    """One of `choices` for each row."""
    at = torch.randint(len(choices), (c["rows"],), generator=g, device="cuda")
    return torch.tensor(choices, dtype=torch.int32 if type(choices[0]) is int else torch.float32, device="cuda")[at]


def _filters(c, g):
    rows, kind = c["rows"], c["filters"]
    full = lambda v: torch.full((rows,), v, dtype=torch.int32 if type(v) is int else torch.float32, device="cuda")  # noqa: E731
    if kind == "usual":
        return dict(temperature=full(0.8), top_k=full(50), top_p=full(0.95))
    if kind == "top_p":
        return dict(top_p=0.85 + 0.1 * torch.rand((rows,), generator=g, device="cuda"))
    if kind == "temperature":
        return dict(temperature=0.6 + torch.rand((rows,), generator=g, device="cuda"))
    if kind == "each":
        return dict(temperature=_rows_of(c, g, [0.0, 0.6, 0.8, 1.0, 1.0, 1.3]), top_k=_rows_of(c, g, [0, 0, 1, 20, 50, 200]),
                    top_p=_rows_of(c, g, [1.0, 1.0, 0.95, 0.9, 0.7]), min_p=_rows_of(c, g, [0.0, 0.0, 0.02, 0.1]))
    return {}


def _prepare_sample(c, g):
    rows, cols, src = c["rows"], c["cols"], c["src"]
    s = dict(uniforms=torch.rand((rows, c["shots"]), generator=g, device="cuda", dtype=torch.float64), filters=_filters(c, g))
    if src == "state":
        a = torch.randn((rows, cols, 2), generator=g, device="cuda")
        s["scores"] = a / a.double().square().sum(dim=(1, 2), keepdim=True).sqrt().float()
    elif src == "probs":
        p = torch.rand((rows, cols), generator=g, device="cuda").log_().neg_().pow_(1.5)
        if c["masked"]:
            p[:, ::3] = 0.0
        s["scores"] = p / p.sum(dim=1, keepdim=True)
    else:
        z = _scores(c, g)
        if c["masked"]:  # outcomes that a grammar forbids, some by the type's lowest value; every seventh row has none left
            z[torch.rand(z.shape, generator=g, device="cuda") < 0.6] = -math.inf
            z[:, ::5] = torch.finfo(FLOATS[src]).min
            z[3::7] = -math.inf
        s["scores"] = z.to(FLOATS[src])[:, :cols]
    s["out"] = torch.zeros((rows, c["shots"]), dtype=torch.int64, device="cuda")
    s["logp"] = torch.zeros((rows, c["shots"]), device="cuda")
    s["kept"] = torch.zeros((rows,), dtype=torch.int32, device="cuda")
    return s


def _prepare_distill(c, g):
    rows, cols, top, t = c["rows"], c["cols"], c["top"], c["temperature"]
    z = _scores(c, g)
    teacher = torch.randn(z.shape, generator=g, device="cuda").mul_(1.5).add_(z, alpha=0.7)[:, :cols]
    logits, at = torch.topk(teacher, top, dim=1)
    at = at.to(torch.int32)
    if top > 4:
        at[1::4, top - top // 4:] = -1  # teachers that gave fewer entries
    at[5::11] = -1                      # positions that are not trained on
    s = dict(scores=z.to(FLOATS[c["src"]])[:, :cols], top_idx=at.contiguous(), top_logits=logits.contiguous(), temperature=t)
    if c["lse"]:
        s["top_lse"] = torch.logsumexp(teacher / t, dim=1)
    del teacher, z
    s["grad_loss"] = (torch.rand((rows,), generator=g, device="cuda") + 0.5) / rows
    s["loss"] = torch.zeros((rows,), device="cuda")
    s["stats"] = torch.zeros((rows, 2), device="cuda")
    if c["what"] == "grad":
        v = s["scores"].float()
        s["stats"][:, 0] = v.amax(dim=1)
        s["stats"][:, 1] = ((v - s["stats"][:, :1]) / t).exp_().sum(dim=1)
    if c["what"] != "loss":
        s["grad"] = torch.zeros((rows, cols), dtype=FLOATS[c["src"]], device="cuda")
    return s


def _handle(c):
    """A context of the library, as a program has it for its circuit."""
    from paper_2602_13140_amd import binding as qb
    if c["op"] == "sample":
        n = c["cols"].bit_length() - 1 if c["src"] == "state" else 1
        batch = c["rows"] if c["src"] == "state" else 1
        need = qb.qsv_sample_workspace_bytes(c["rows"], c["cols"])
    else:
        n, batch, need = 1, 1, qb.qsv_distill_workspace_bytes(c["rows"], c["cols"])
    return qb.Context(n, batch, ws_bytes=max(need, qb.qsv_workspace_bytes(n, batch)))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(6007 * int(seed) + 29)
    s = _prepare_sample(case, g) if case["op"] == "sample" else _prepare_distill(case, g)
    s["case"] = case
    if own:
        s["ctx"] = _handle(case)
        if case.get("src") == "state":
            s["ctx"].state.copy_(s["scores"])
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _values(s):
    """Values that order the outcomes, and which of them there are: scores, or probabilities as QSV_M_PROBS writes them."""
    src = s["case"]["src"]
    if src == "state":  # re^2 rounded, then im^2 added with one rounding
        re, im = s["scores"][..., 0], s["scores"][..., 1]
        v = (im.double().square() + (re * re).double()).float()
        return v, v > 0
    if src == "probs":
        return s["scores"], s["scores"] > 0
    v = s["scores"].float() + 0.0
    return v, v > -math.inf


def _plain_sample(s):
    """In 64 bits: outcomes are whole numbers, decided at borders of running sums."""
    f, logs = s["filters"], s["case"]["src"] in FLOATS
    v, there = _values(s)
    rows, cols = v.shape
    v = torch.where(there, v, torch.full_like(v, -math.inf))
    v, order = torch.sort(v, dim=1, descending=True, stable=True)
    there = torch.gather(there, 1, order)
    off = lambda name, value: f[name].view(-1, 1) if name in f else torch.full((rows, 1), value, device=v.device)  # noqa: E731
    t, top_k, top_p, min_p = off("temperature", 1.0), off("top_k", 0), off("top_p", 1.0), off("min_p", 0.0)
    m, d = v[:, :1].double(), v.double()
    t64 = torch.where(t > 0, t, torch.ones_like(t)).double()
    e = torch.exp((d - m) / t64) if logs else torch.where(t64 == 1, d / m, torch.exp(torch.log(d / m) / t64))
    e = torch.where(there, torch.where(d == m, torch.ones_like(e), e), torch.zeros_like(e))
    place = torch.arange(cols, device=v.device).view(1, -1)
    keep = there & (e >= min_p.double())
    keep &= (top_k == 0) | (place < top_k)
    keep &= (t > 0) | (place == 0)
    bits = min(51, 62 - (cols - 1).bit_length())
    w = torch.where(keep, torch.round(e * 2.0 ** bits).to(torch.int64), 0)
    total = w.sum(dim=1, keepdim=True)
    part = torch.round(top_p.double().clamp(max=1.0) * 2.0 ** 31).to(torch.int64)
    low = part * (total & (2 ** 31 - 1))
    border = part * (total >> 31) + (low >> 31) + ((low & (2 ** 31 - 1)) != 0)
    keep &= (top_p >= 1) | (torch.cumsum(w, dim=1) - w < border) | (place == 0)
    w = torch.where(keep, w, 0)
    by_index = torch.zeros_like(w).scatter_(1, order, w)
    run = torch.cumsum(by_index, dim=1)
    total = run[:, -1:]
    r = torch.floor(s["uniforms"] * 2.0 ** 53).to(torch.int64)
    r1, r0, w1, w0 = r >> 27, r & (2 ** 27 - 1), total >> 32, total & (2 ** 32 - 1)   # floor(r total / 2^53) in parts
    at = r1 * w1 * 64 + ((((r0 * w0) >> 27) + r1 * w0 + r0 * w1 * 32) >> 26)
    out = torch.searchsorted(run, at, right=True)
    some = total > 0
    out = torch.where(some, out, 0)
    logp = torch.log(torch.gather(by_index, 1, out).double() / total.double())
    logp = torch.where(some, logp, torch.full_like(logp, -math.inf))
    return {"out": torch.where(some, out, -1), "logp": logp.float(), "kept": keep.sum(dim=1).to(torch.int32)}


def _teacher(s, cols):
    """q of every entry (0 where there is none) and the place it belongs to."""
    at, t = s["top_idx"].long(), s["temperature"]
    real = (at >= 0) & (at < cols)
    x = torch.where(real, s["top_logits"].double() / t, -math.inf)
    if "top_lse" in s:
        q = torch.exp(x - s["top_lse"].double().view(-1, 1))
    else:
        high = x.amax(dim=1, keepdim=True)
        e = torch.exp(x - torch.where(high > -math.inf, high, 0.0))
        q = e / e.sum(dim=1, keepdim=True).clamp(min=1e-300)
    return q, torch.where(real, at, 0)


def _plain_distill(s):
    z, t, what = s["scores"].float(), s["temperature"], s["case"]["what"]
    q, at = _teacher(s, z.shape[1])
    m = s["stats"][:, :1] if what == "grad" else z.amax(dim=1, keepdim=True)
    e = torch.exp((z - m) / t)
    total = s["stats"][:, 1:] if what == "grad" else e.sum(dim=1, keepdim=True)
    got = {}
    if what != "grad":
        lnp = (torch.gather(z, 1, at).double() - m.double()) / t - torch.log(total.double())
        got["loss"] = torch.where(q > 0, q * (torch.log(q) - lnp), 0.0).sum(dim=1).float()
    if what == "loss":
        got["stats"] = torch.cat((m, total), dim=1)
    else:
        grad = e * (q.sum(dim=1, keepdim=True).float() / total)
        grad.scatter_add_(1, at, -q.float())
        got["grad"] = (grad * (s["grad_loss"].view(-1, 1) / t)).to(s["scores"].dtype)
    return got


# ---- one pass --------------------------------------------------------------------------------------------------------
def _own_sample(s):
    from paper_2602_13140_amd import binding as qb
    src = s["case"]["src"]
    kind = {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16, "probs": qb.QSV_S_PROBS, "state": qb.QSV_S_STATE}[src]
    s["ctx"].qsv_sample(kind, s["out"], s["uniforms"], scores=None if src == "state" else s["scores"], logp=s["logp"],
                        kept=s["kept"], **s["filters"])
    return {k: s[k] for k in ("out", "logp", "kept")}


def _own_distill(s):
    from paper_2602_13140_amd import binding as qb
    what = s["case"]["what"]
    kind = {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16}[s["case"]["src"]]
    s["ctx"].qsv_distill(kind, s["scores"], s["top_idx"], s["top_logits"], s["temperature"], top_lse=s.get("top_lse"),
                         loss=None if what == "grad" else s["loss"], stats=None if what == "both" else s["stats"],
                         have_stats=int(what == "grad"), grad_loss=None if what == "loss" else s["grad_loss"], grad=s.get("grad"))
    return {k: s[k] for k in {"both": ("loss", "grad"), "loss": ("loss", "stats"), "grad": ("grad",)}[what]}


def run(s):
    if s["case"]["op"] == "sample":
        return _own_sample(s) if own else _plain_sample(s)
    return _own_distill(s) if own else _plain_distill(s)


def work(case):
    """Scores read once, results written once; a subtraction, a product, an exponential and a sum for each score (and, for a
    gradient, a product and a difference more)."""
    c = case
    n = c["rows"] * c["cols"]
    size = BYTES[c["src"]]
    if c["op"] == "sample":
        return {"bytes": n * size + c["rows"] * (c["shots"] * 20 + 20), "flops": 4 * n}
    teacher = c["rows"] * c["top"] * 8
    if c["what"] == "loss":
        return {"bytes": n * size + teacher + c["rows"] * 16, "flops": 4 * n}
    return {"bytes": 2 * n * size + teacher + c["rows"] * 16, "flops": 6 * n}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------
def _exact_row(v, logs, cols, t, top_k, top_p, min_p, uniforms):
    """(outcomes, ln of their probabilities, outcomes left) of one row; masked values are -inf (scores) or 0."""
    nothing = [-1] * len(uniforms), [-math.inf] * len(uniforms), 0
    v = v.astype(np.float64)
    left = np.flatnonzero(v > (-math.inf if logs else 0.0))
    if not left.size:
        return nothing
    left = left[np.argsort(-v[left], kind="stable")]
    top = v[left[0]]
    if t == 0:
        left = left[:1]
    with np.errstate(divide="ignore", invalid="ignore", over="ignore", under="ignore"):
        e = np.exp((v[left] - top) / t) if logs and t > 0 else (v[left] / top if t in (0, 1) else (v[left] / top) ** (1.0 / t))
    e = np.where(v[left] == top, 1.0, e)
    left, e = left[e >= min_p], e[e >= min_p]
    if top_k > 0:
        left, e = left[:top_k], e[:top_k]
    scale = 2.0 ** min(51, 62 - (cols - 1).bit_length())
    w = np.rint(e * scale).astype(np.int64)
    if top_p < 1:
        mass = -(-int(round(top_p * 2 ** 31)) * int(w.sum()) // 2 ** 31)
        n = max(1, int(np.searchsorted(np.cumsum(w) - w, mass, side="left")))
        left, w = left[:n], w[:n]
    kept = len(left)
    by = np.argsort(left)
    left, w = left[by], w[by]
    run = np.cumsum(w)
    total = int(run[-1])
    at = np.array([math.floor(u * 2 ** 53) * total >> 53 for u in uniforms], dtype=np.int64)
    hit = np.searchsorted(run, at, side="right")
    return left[hit], np.log(w[hit].astype(np.float64) / total), kept


def _exact_sample(s):
    c, f = s["case"], s["filters"]
    a = s["scores"].float().cpu().numpy() if c["src"] != "state" else s["scores"].cpu().numpy()
    if c["src"] == "state":
        a = (a[..., 1].astype(np.float64) ** 2 + np.float32(a[..., 0] * a[..., 0]).astype(np.float64)).astype(np.float32)
    u = s["uniforms"].cpu().numpy().tolist()
    of = {k: x.double().cpu().tolist() for k, x in f.items()}
    got = []
    for r in range(c["rows"]):
        p = [of[k][r] if k in of else d for k, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))]
        got.append(_exact_row(a[r], c["src"] in FLOATS, c["cols"], p[0], int(p[1]), p[2], p[3], u[r]))
    return {"out": np.array([x[0] for x in got], dtype=np.int64), "logp": np.array([x[1] for x in got], dtype=np.float64),
            "kept": np.array([x[2] for x in got], dtype=np.int32)}


def _exact_distill(s):
    """A part of the rows at a time."""
    c, t = s["case"], s["temperature"]
    rows, cols, what = c["rows"], c["cols"], c["what"]
    got = {}
    step = max(1, (1 << 26) // cols)
    for b in range(0, rows, step):
        z = s["scores"][b:b + step].double()
        at = s["top_idx"][b:b + step].long()
        real = ((at >= 0) & (at < cols)).double()
        at = at.clamp(0, cols - 1)
        x = s["top_logits"][b:b + step].double() / t
        norm = s["top_lse"][b:b + step, None].double() if "top_lse" in s else torch.log((real * torch.exp(x - x[:, :1])).sum(1, True)) + x[:, :1]
        q = torch.where(real > 0, torch.exp(x - norm), 0.0)
        if what == "grad":
            lse = s["stats"][b:b + step, :1].double() / t + torch.log(s["stats"][b:b + step, 1:].double())
        else:
            lse = torch.logsumexp(z / t, dim=1, keepdim=True)
        now = {}
        if what != "grad":
            now["loss"] = torch.where(q > 0, q * (torch.log(q) - torch.gather(z, 1, at) / t + lse), 0.0).sum(1)
        if what == "loss":
            m = z.amax(1, True)
            now["stats"] = torch.cat((m, torch.exp(lse - m / t)), 1)
        else:
            grad = torch.exp(z / t - lse) * q.sum(1, True)
            grad.scatter_add_(1, at, -q)
            now["grad"] = grad * s["grad_loss"][b:b + step, None].double() / t
        for k, y in now.items():
            got.setdefault(k, []).append(y)
    return {k: torch.cat(y) for k, y in got.items()}


def exact(case, seed):
    global own
    was, own = own, False        # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _exact_sample(s) if case["op"] == "sample" else _exact_distill(s)
