"""qsv_adjust and qsv_adjust_grad against their formulas in 64 bits.

Errors that the kernels may make:
  a place with a word (history or entries)  worked out in float64 and rounded to the type once: half a step; the float64 sums are off by
        2^-50 of their largest term at most (six roundings)
  another place with a shared bias          one sum in float32, 2^-24, then the type: half a step; without one nothing is rounded
  gradients of scores                       as a place with a word: 1 / R and the product, 2^-51
  d / d b                                   sums in float64 (up to 2^12 of them: 2^-40 of the absolute sum), one rounding to float32
  d / d e                                   the value itself: exact
Every rounding to the type may miss by half its smallest number below its normal range."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2602_13140_amd import binding as qb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF, NAN = math.inf, math.nan
U = 2.0 ** -24
KIND = {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16}


def tt(src):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[src]


# ---- the formulas ----------------------------------------------------------------------------------------------------
def facts(q, r, cols):
    """s, c and a of row r (a None: its parameters are out of range)."""
    get = lambda k, d: d if q.get(k) is None else q[k][r]  # noqa: E731
    by, each, once = (float(get(k, d)) for k, d in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0)))
    ok = by > 0 and by < INF and abs(each) < INF and abs(once) < INF
    s, c = np.zeros(cols, bool), np.zeros(cols)
    if q.get("prior") is not None:
        prior = q["prior"][r]
        length, prompt = int(get("prior_len", len(prior))), int(get("prompt_len", 0))
        ok = ok and 0 <= prompt <= length <= len(prior)
        if ok:
            for i, k in enumerate(prior[:length]):
                if 0 <= k < cols:
                    s[k] = True
                    c[k] += i >= prompt
    allowed = np.ones(cols, bool)
    if q.get("masks") is not None:
        n = len(q["masks"])
        at = int(q["mask_of"][r]) if q.get("mask_of") is not None else (r if n > 1 else 0)
        ok = ok and -1 <= at < n
        if ok and at >= 0:
            k = np.arange(cols)
            allowed = (q["masks"][at].astype(np.int64)[k // 32] >> (k % 32)) & 1 == 1
    return s, c, allowed if ok else None, by, each, once


def forward(z, q):
    """(values, the largest term in them, places that are worked out in float64) of float64 scores z."""
    rows, cols = z.shape
    out, big, word = np.zeros_like(z), np.zeros_like(z), np.zeros(z.shape, bool)
    for r in range(rows):
        s, c, a, by, each, once = facts(q, r, cols)
        if a is None:
            out[r] = NAN
            continue
        with np.errstate(all="ignore"):
            v = np.where(s, np.where(z[r] > 0, z[r] / by, z[r] * by), z[r])
            big[r] = np.maximum(np.abs(v), np.abs(z[r]))
            v = v - (each * c + once * (c > 0))
            big[r] = np.maximum(big[r], abs(each) * c + abs(once))
            if q.get("bias") is not None:
                v = v + q["bias"].astype(np.float64)
                big[r] = np.maximum(big[r], np.abs(q["bias"]))
            word[r] = s
            if q.get("entry_idx") is not None:
                e = np.zeros(cols)
                for k, x in zip(q["entry_idx"][r], q["entry_bias"][r]):
                    if 0 <= k < cols:
                        e[k] += float(x)
                        word[r, k] = True
                v = np.where(word[r], v + e, v)
                big[r] = np.maximum(big[r], np.abs(e))
        out[r] = np.where(a, v, -INF)
    return out, big, word


def backward(z, G, q):
    """(d / d z, d / d b, its absolute sums, d / d e)."""
    rows, cols = G.shape
    grad, n = np.zeros_like(G), 0 if q.get("entry_idx") is None else q["entry_idx"].shape[1]
    db, ab, de = np.zeros(cols), np.zeros(cols), np.zeros((rows, n))
    for r in range(rows):
        s, _, a, by, _, _ = facts(q, r, cols)
        if a is None:
            grad[r], de[r] = NAN, NAN
            db += NAN
            continue
        g = np.where(a, G[r], 0.0)
        grad[r] = np.where(s & a, np.where(z[r] > 0, g / by, g * by), g)
        with np.errstate(invalid="ignore"):
            db += g
        ab += np.abs(g)
        for j in range(n):
            k = q["entry_idx"][r, j]
            de[r, j] = g[k] if 0 <= k < cols else 0.0
    return grad, db, ab, de


def settings(rows, cols, seed, prior=0, entries=0, masks=0, bias=False):
    """Everything at random: repeated and padded outcomes, entries that name the same outcome, masks of which one leaves nothing."""
    g = np.random.default_rng(seed)
    q = {}
    if prior:
        q["prior"] = (g.random((rows, prior)) ** 3 * (cols + 1)).astype(np.int32) - (g.random((rows, prior)) < 0.05)
        q["prior_len"] = g.integers(0, prior + 1, rows).astype(np.int32)
        q["prior_len"][0] = prior
        q["prompt_len"] = (g.random(rows) * (q["prior_len"] + 1)).astype(np.int32)
        q["repetition"] = g.choice(np.float32([1.0, 1.1, 1.3, 0.7]), rows)
        q["frequency"] = g.choice(np.float32([0.0, 0.3, -0.2]), rows)
        q["presence"] = g.choice(np.float32([0.0, 0.5]), rows)
    if entries:
        q["entry_idx"] = g.integers(-1, cols + 1, (rows, entries)).astype(np.int32)
        q["entry_idx"][:, entries // 2:] = q["entry_idx"][:, :entries - entries // 2]
        if prior:
            q["entry_idx"][:, 0] = q["prior"][:, 0]
        q["entry_bias"] = (g.standard_normal((rows, entries)) * 3).astype(np.float32)
    if masks:
        words = (cols + 31) // 32 + 1
        q["masks"] = g.integers(0, 2 ** 32, (masks, words), dtype=np.uint32)
        q["masks"][-1] = 0
        if masks > 1:
            q["masks"][0, :words // 2] = 0xffffffff
        q["mask_of"] = g.integers(-1, masks, rows).astype(np.int32)
    if bias:
        q["bias"] = g.standard_normal(cols).astype(np.float32)
    return q


def forward_all(z, q):
    """forward, of all rows at once; its allowed places too."""
    rows, cols = z.shape
    get = lambda k, d: np.full(rows, d) if q.get(k) is None else q[k].astype(np.float64)  # noqa: E731
    by, each, once = get("repetition", 1.0), get("frequency", 0.0), get("presence", 0.0)
    good = (by > 0) & (by < INF) & (np.abs(each) < INF) & (np.abs(once) < INF)
    s, c, e, word = np.zeros(z.shape, bool), np.zeros(z.shape), np.zeros(z.shape), np.zeros(z.shape, bool)
    at = lambda k, on: np.flatnonzero(on) // k.shape[1] * cols + k[on]  # noqa: E731
    if q.get("prior") is not None:
        prior, place = q["prior"].astype(np.int64), np.arange(q["prior"].shape[1])
        length, prompt = get("prior_len", float(len(place))), get("prompt_len", 0.0)
        good &= (prompt >= 0) & (prompt <= length) & (length <= len(place))
        real = (prior >= 0) & (prior < cols) & (place < length[:, None])
        s.flat[at(prior, real)] = True
        c += np.bincount(at(prior, real & (place >= prompt[:, None])), minlength=z.size).reshape(z.shape)
        word |= s
    if q.get("entry_idx") is not None:
        idx = q["entry_idx"].astype(np.int64)
        real = (idx >= 0) & (idx < cols)
        e += np.bincount(at(idx, real), weights=q["entry_bias"][real].astype(np.float64), minlength=z.size).reshape(z.shape)
        word.flat[at(idx, real)] = True
    a = np.ones(z.shape, bool)
    if q.get("masks") is not None:
        bits = np.unpackbits(q["masks"].view(np.uint8), axis=1, bitorder="little")[:, :cols] == 1
        a = bits[q["mask_of"]] | (q["mask_of"] < 0)[:, None]
    b = np.zeros(cols) if q.get("bias") is None else q["bias"].astype(np.float64)
    with np.errstate(divide="ignore"):
        v = np.where(s, np.where(z > 0, z / by[:, None], z * by[:, None]), z)
    less = each[:, None] * c + once[:, None] * (c > 0)
    most = np.abs(each)[:, None] * c + np.abs(once)[:, None]
    big = np.max([np.abs(v), np.abs(z), most, np.broadcast_to(np.abs(b), z.shape), np.abs(e)], axis=0)
    v = np.where(a, v - less + b + e, -INF)
    return np.where(good[:, None], v, NAN), big, word, s, a, good


def backward_all(z, G, q):
    """backward, of all rows at once and without the entries."""
    _, _, _, s, a, good = forward_all(z, q)
    by = (np.ones(len(z)) if q.get("repetition") is None else q["repetition"].astype(np.float64))[:, None]
    g = np.where(good[:, None], np.where(a, G, 0.0), NAN)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.where(s & a, np.where(z > 0, g / by, g * by), g), g.sum(0), np.abs(g).sum(0)


def test_all_rows_at_once_as_one_by_one():
    g = np.random.default_rng(4)
    for seed, (rows, cols, prior, entries, masks, bias) in enumerate([(9, 40, 30, 6, 4, True), (5, 3, 9, 0, 2, False), (7, 70, 0, 5, 0, True), (6, 33, 12, 0, 3, False)]):
        z, G, q = g.standard_normal((rows, cols)) * 3, g.standard_normal((rows, cols)), settings(rows, cols, seed, prior, entries, masks, bias)
        if prior:
            q["prompt_len"][1], q["repetition"][2] = q["prior_len"][1] + 1, -1.0
        v, big, word = forward(z, q)
        got = forward_all(z, q)
        ok = got[5]
        assert (~ok).sum() == (2 if prior else 0) and np.allclose(got[0], v, rtol=1e-14, atol=1e-14, equal_nan=True)
        assert np.array_equal(got[2][ok], word[ok]) and np.allclose(got[1][ok], big[ok], rtol=1e-14)
        grad, db, ab = backward_all(z, G, q)
        want = backward(z, G, q)
        assert np.allclose(grad, want[0], rtol=1e-14, equal_nan=True) and np.allclose(db, want[1], rtol=1e-14, atol=1e-13, equal_nan=True)
        assert not ok.all() or np.allclose(ab, want[2], rtol=1e-14, atol=1e-13)


def test_gradients_against_differences():
    g = np.random.default_rng(3)
    rows, cols, h = 4, 9, 1e-6
    z, G = g.standard_normal((rows, cols)) * 2, g.standard_normal((rows, cols))
    q = settings(rows, cols, 5, prior=6, entries=4, masks=3, bias=True)
    for k in ("bias", "entry_bias"):
        q[k] = q[k].astype(np.float64)
    grad, db, _, de = backward(z, G, q)

    def loss(z, q):
        v = forward(z, q)[0]
        return np.where(v > -INF, G * np.where(v > -INF, v, 0.0), 0.0).sum()
    for r in range(rows):
        for k in range(cols):
            step = np.zeros_like(z)
            step[r, k] = h
            assert abs((loss(z + step, q) - loss(z - step, q)) / (2 * h) - grad[r, k]) < 1e-7
        for j in range(4):
            up, down = q["entry_bias"].copy(), q["entry_bias"].copy()
            up[r, j] += h
            down[r, j] -= h
            assert abs((loss(z, dict(q, entry_bias=up)) - loss(z, dict(q, entry_bias=down))) / (2 * h) - de[r, j]) < 1e-7
    for k in range(cols):
        step = np.zeros(cols)
        step[k] = h
        assert abs((loss(z, dict(q, bias=q["bias"] + step)) - loss(z, dict(q, bias=q["bias"] - step))) / (2 * h) - db[k]) < 1e-7


# ---- refusals, without a device --------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    lib = str(tmp_path_factory.mktemp("checks") / "lists.so")
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-fsanitize=undefined", "-static-libubsan",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2602_13140_amd", "csrc"),
                           os.path.join(ROOT, "tests", "check_lists.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    for f, n in ((L.request_adjust, 1), (L.request_adjust_grad, 2)):
        f.restype = ctypes.c_char_p
        f.argtypes = [ctypes.c_void_p] * n
    return L


def req(**more):
    r = qb.qsv_adjust_req()
    r.kind, r.scores_dev, r.rows, r.cols, r.row_stride = qb.QSV_S_BF16, 0x10000, 3, 40, 48
    r.out_dev, r.out_stride = 0x20000, 40
    for k, v in more.items():
        setattr(r, k, v)
    return r


def back(**more):
    b = qb.qsv_adjust_grad_req(0x40000, 40, 0x50000, 44, 0x60000, None)
    for k, v in more.items():
        setattr(b, k, v)
    return b


def test_refusals(checks):
    def say(**more):
        return checks.request_adjust(ctypes.byref(req(**more)))
    assert say() is None and b"req" in checks.request_adjust(None)
    for kind in (0, qb.QSV_S_PROBS, qb.QSV_S_STATE, 9):
        assert b"kind" in say(kind=kind)
    assert b"rows" in say(rows=-1) and b"cols" in say(cols=0) and b"cols" in say(cols=2 ** 30 + 1) and b"row_stride" in say(row_stride=39)
    assert say(rows=0, scores_dev=None, out_dev=None) is None
    assert b"scores_dev" in say(scores_dev=None) and b"NULL" in say(out_dev=None)
    assert b"aligned" in say(scores_dev=0x10001) and b"aligned" in say(out_dev=0x20001) and b"stride" in say(out_stride=39)
    assert say(out_dev=0x10000, out_stride=48) is None                                    # over the scores
    assert b"overlap" in say(out_dev=0x10000) and b"overlap" in say(out_dev=0x10002, out_stride=48)
    assert say(out_dev=0x10000 + (2 * 48 + 40) * 2) is None and b"overlap" in say(out_dev=0x10000 + (2 * 48 + 40) * 2 - 2)
    assert say(rows=1, out_dev=0x10000, out_stride=0, row_stride=0) is None
    assert b"n_prior" in say(n_prior=-1) and b"n_prior" in say(n_prior=2 ** 20 + 1) and b"prior_dev" in say(n_prior=4)
    assert b"prior_stride" in say(n_prior=4, prior_dev=0x1000, prior_stride=3) and say(n_prior=4, prior_dev=0x1000, prior_stride=4) is None
    assert b"n_entries" in say(n_entries=-1) and b"n_entries" in say(n_entries=1024)
    assert b"entry" in say(n_entries=2) and b"entry" in say(n_entries=2, entry_idx_dev=0x1000)
    assert say(n_entries=1023, entry_idx_dev=0x1000, entry_bias_dev=0x3000) is None
    m = dict(masks_dev=0x1000, mask_stride=2)
    assert say(n_masks=1, **m) is None and say(n_masks=3, **m) is None and b"n_masks" in say(n_masks=0, **m)
    assert b"mask_of" in say(n_masks=2, **m) and say(n_masks=2, mask_of_dev=0x2000, **m) is None
    assert b"mask_stride" in say(n_masks=3, masks_dev=0x1000, mask_stride=1) and say(n_masks=1, masks_dev=0x1000, mask_stride=0) is None
    assert qb.load().qsv_adjust(None, ctypes.byref(req())) == qb.QSV_ERR_INVALID_ARG


def test_refusals_of_the_backward_pass(checks):
    def say(r=None, **more):
        return checks.request_adjust_grad(ctypes.byref(req(**(r or {}))), ctypes.byref(back(**more)))
    assert say() is None and b"NULL" in checks.request_adjust_grad(ctypes.byref(req()), None) and b"NULL" in checks.request_adjust_grad(None, ctypes.byref(back()))
    assert say(r=dict(scores_dev=None, out_dev=None)) is None
    history = dict(n_prior=4, prior_dev=0x1000, prior_stride=4, repetition_dev=0x2000)
    assert say(r=history) is None and b"scores_dev" in say(r=dict(history, scores_dev=None)) and say(r=dict(history, scores_dev=None), grad_dev=None) is None
    assert b"overlap the scores" in say(r=history, grad_dev=0x10000, grad_stride=48) and say(grad_dev=0x10000, grad_stride=48) is None
    assert b"kind" in say(r=dict(kind=4)) and b"rows" in say(r=dict(rows=-1))
    assert b"NULL" in say(grad_out_dev=None) and b"aligned" in say(grad_out_dev=0x40001) and b"stride" in say(grad_out_stride=39)
    assert b"aligned" in say(grad_dev=0x50001) and b"stride" in say(grad_stride=39)
    assert b"overlap" in say(grad_dev=0x40000) and say(grad_dev=0x40000, grad_stride=40) is None
    assert b"entries" in say(grad_entry_dev=0x7000) and say(r=dict(n_entries=2, entry_idx_dev=0x1000), grad_entry_dev=0x7000) is None
    assert say(r=dict(rows=0), grad_out_dev=None, grad_dev=None) is None
    assert qb.load().qsv_adjust_grad(None, ctypes.byref(req()), ctypes.byref(back())) == qb.QSV_ERR_INVALID_ARG


def test_layouts():
    assert [ctypes.sizeof(x) for x in (qb.qsv_adjust_req, qb.qsv_adjust_grad_req)] == [176, 48]
    assert qb.qsv_adjust_grad_workspace_bytes(-1, 5) == 0 == qb.qsv_adjust_grad_workspace_bytes(5, 0)
    assert 0 < qb.qsv_adjust_grad_workspace_bytes(0, 1) <= qb.qsv_adjust_grad_workspace_bytes(4096, 131072)


def test_tensors_that_the_binding_refuses():
    """On the host (device -1), as every refusal is raised."""
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    ok = dict(prior=i32(3, 4), prior_len=i32(3), prompt_len=i32(3), repetition=torch.ones(3), frequency=torch.ones(3), presence=torch.ones(3),
              entry_idx=i32(3, 2), masks=i32(5, 2), mask_of=i32(3))

    def take(**more):
        r = qb.qsv_adjust_req()
        r.cols = 40
        qb._adjustment(r, -1, 3, **dict(ok, **more))
        return r
    r = take()
    assert (r.n_prior, r.prior_stride, r.n_entries, r.n_masks, r.mask_stride) == (4, 4, 2, 5, 2)
    assert take(prior=i32(3, 8)[:, 1:5]).prior_stride == 8 and take(prior=i32(3, 0)).n_prior == 0
    for bad in (dict(prior=i32(2, 4)), dict(prior=i32(4)), dict(prior=i32(4, 3).t()), dict(prior=ok["prior"].long()), dict(prior_len=i32(2)),
                dict(prompt_len=torch.zeros(3)), dict(repetition=torch.ones(3).double()), dict(presence=torch.ones(3, 1)), dict(entry_idx=i32(3)),
                dict(entry_idx=i32(4, 2)), dict(masks=i32(5, 1)), dict(masks=i32(5)), dict(mask_of=i32(5)), dict(masks=None)):
        with pytest.raises(qb.QsvError) as e:
            take(**bad)
        assert e.value.status == qb.QSV_ERR_INVALID_ARG


# ---- on the GPU ------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ctx():
    c = qb.Context(1, 1)
    yield c
    c.close()


def dev(q):
    import torch
    got = {}
    for k, a in q.items():
        if a is not None:
            got[k] = torch.from_numpy(np.ascontiguousarray(a).view(np.int32) if a.dtype == np.uint32 else np.ascontiguousarray(a)).cuda()
    return got


def f64(t):
    return t.double().cpu().numpy()


def draw(src, rows, cols, seed, pad=0, sigma=4.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, cols + pad), generator=g) * sigma).to(tt(src)).cuda()[:, :cols]


def close(src, got, want, tol):
    """Within tol, and the rounding to the type; infinite and NaN places the same."""
    import torch
    f = torch.finfo(tt(src))
    with np.errstate(all="ignore"):
        over = np.abs(want) >= f.max * (1 + f.eps / 4)             # rounds to infinity
        want = np.where(over, np.sign(want) * INF, want)
        edge = np.abs(np.abs(want) / f.max - 1) < f.eps            # may go either way after an error of tol
        half = np.maximum(f.eps / 2 * np.abs(want), f.smallest_normal * f.eps / 2)
        ok = (np.abs(got - want) <= (half + tol) * (1 + f.eps) + 2.0 ** -149) | (got == want) | (np.isnan(want) & np.isnan(got)) | (edge & (tol > 0))
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


def check_forward(ctx, src, z, q, over=False, pad=0):
    import torch
    want, big, word = forward(f64(z), q)
    rows, cols = z.shape
    whole = torch.full((rows, cols + pad), 55.0, dtype=tt(src), device="cuda")
    if over:
        whole[:, :cols] = z
    out, keep = whole[:, :cols], z.clone()
    ctx.qsv_adjust(KIND[src], out if over else z, None if over else out, **dev(q))
    torch.cuda.synchronize()
    assert np.array_equal(f64(z), f64(keep), equal_nan=True)
    if pad:
        assert bool((whole[:, cols:] == 55.0).all())
    with np.errstate(all="ignore"):
        tol = np.where(word, 2.0 ** -50 * big, U * np.abs(want) if q.get("bias") is not None and src != "f32" else 0.0)
    close(src, f64(out), want, np.nan_to_num(tol, nan=0.0, posinf=0.0))
    return out


def check_backward(ctx, src, z, G, q, over=False, pad=0, bias=True, grad=True):
    import torch
    want, db, ab, de = backward(f64(z), f64(G), q)
    rows, cols = G.shape
    q = {k: x for k, x in q.items() if k not in ("bias", "entry_bias")}
    whole = torch.full((rows, cols + pad), 55.0, dtype=tt(src), device="cuda")
    if over:
        whole[:, :cols] = G
    out = whole[:, :cols]
    b = torch.full((cols,), 77.0, device="cuda") if bias else None
    e = torch.full(q["entry_idx"].shape, 77.0, device="cuda") if "entry_idx" in q else None
    ctx.qsv_adjust_grad(KIND[src], out if over else G, grad=out if grad else None, scores=z, grad_bias=b, grad_entry=e, **dev(q))
    torch.cuda.synchronize()
    if pad:
        assert bool((whole[:, cols:] == 55.0).all())
    if grad:
        close(src, f64(out), want, np.where(np.isfinite(want), 2.0 ** -50 * np.abs(want), 0.0))
    if bias:
        got = f64(b)
        assert ((np.abs(got - db) <= U * np.abs(db) + 2.0 ** -40 * ab + 2.0 ** -149) | (np.isnan(got) & np.isnan(db))).all()
    if e is not None:
        assert np.array_equal(f64(e), de, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [1, 2, 7, 31, 33, 64, 255, 1000, 2049, 4099, 8192, 8193, 16391, 33001, 70001])
def test_sizes(ctx, src, cols):
    rows = 5
    for n, (prior, entries, masks, bias, pad) in enumerate([(0, 0, 0, False, 0), (0, 0, 3, False, 1), (1, 0, 0, False, 0), (9, 3, 2, True, 3),
                                                           (700, 40, 4, False, 8), (0, 1, 1, True, 0), (300, 0, 0, True, 1)]):
        z, q = draw(src, rows, cols, 10 * cols + n, pad), settings(rows, cols, cols + n, prior, entries, masks, bias)
        check_forward(ctx, src, z, q, pad=pad)
        check_forward(ctx, src, z, q, over=True, pad=pad)
        G = draw(src, rows, cols, 11 * cols + n, pad, sigma=0.3)
        for over in (False, True):
            check_backward(ctx, src, z, G, q, over, pad, bias=bias or n == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,prior", [(1, 200003, 5000), (1, 32768, 700), (130, 9000, 64), (513, 300, 20), (1030, 77, 5), (2, 3000, 40000),
                                             (300, 33000, 128), (70, 65536, 300)])
def test_rows_and_histories(ctx, src, rows, cols, prior):
    z, q = draw(src, rows, cols, rows), settings(rows, cols, rows, prior, 17, 5, rows % 2 == 0)
    if rows == 1:
        q["mask_of"][:] = 0
    check_forward(ctx, src, z, q)
    check_forward(ctx, src, z, q, over=True)
    G = draw(src, rows, cols, rows + 1, sigma=0.1)
    check_backward(ctx, src, z, G, q, bias=False)
    check_backward(ctx, src, z, G, q, over=True)
    check_backward(ctx, src, z, G, q, grad=False)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,prior,entries", [
    (700, 200, 30, 5),          # a wavefront's row
    (700, 1500, 2048, 0), (600, 1900, 90, 9), (600, 3600, 700, 2), (520, 9100, 1000, 1023),     # short rows and longer ones, kept histories
    (520, 6000, 2049, 3), (257, 33000, 9000, 1000), (300, 33000, 5000, 1023),                                             # the largest parts, kept and not
    (3, 20000, 2048, 1023), (3, 20000, 2049, 40), (3, 20000, 8193, 1023), (5, 70000, 4000, 96), (5, 70000, 4097, 0)])
def test_every_way_through(ctx, src, rows, cols, prior, entries):
    z, q = draw(src, rows, cols, rows + cols), settings(rows, cols, rows, prior, entries, 3, rows % 2 == 1)
    G = draw(src, rows, cols, rows + 2, sigma=0.2)
    check_forward(ctx, src, z, q, over=False)
    check_forward(ctx, src, z, dict(q, bias=None), over=True)
    if rows % 2:
        check_forward(ctx, src, z, q, over=True)
    check_backward(ctx, src, z, G, q, bias=False)
    check_backward(ctx, src, z, G, q, over=True)
    check_backward(ctx, src, z, G, q, over=True, bias=False)


@pytest.mark.gpu
@pytest.mark.parametrize("src,rows,cols", [("f32", 5, 500), ("f16", 4, 70), ("bf16", 3, 1024), ("f32", 3, 3), ("bf16", 520, 33)])
@pytest.mark.parametrize("prior", [255, 256, 257, 2047, 2048, 2049, 20000])
def test_short_rows_with_long_histories(ctx, src, rows, cols, prior):
    """More earlier outcomes than columns: with the threads that keep them and the passes that do not, few rows and many."""
    if rows > 5 and prior > 2049:
        prior = 3000
    z, q = draw(src, rows, cols, rows + prior), settings(rows, cols, prior, prior, 6, 2, rows % 2 == 1)
    G = draw(src, rows, cols, rows + 3, sigma=0.2)
    check_forward(ctx, src, z, q, pad=1)
    check_backward(ctx, src, z, G, q, bias=False)
    if rows <= 5:
        check_forward(ctx, src, z, dict(q, bias=None), over=True)
        check_backward(ctx, src, z, G, q, over=True)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [50, 9000])
def test_values_at_the_ends_of_the_type(ctx, src, cols):
    """-inf, +inf, NaN and the lowest value, masked and not, in rows of history and without; biases that exclude."""
    import torch
    rows, low = 8, torch.finfo(tt(src)).min
    z = draw(src, rows, cols, 1).clone()
    z[:, 0], z[:, 1], z[:, 2], z[:, 3], z[:, 4], z[:, 5] = -INF, INF, NAN, low, -low, 0.0
    z[1] = -INF
    z[2] = low
    z[3] = NAN
    q = settings(rows, cols, 4, prior=30, entries=6, masks=4, bias=True)
    q["prior"][:, :8] = np.arange(8)
    q["prior_len"][:] = [30, 30, 30, 30, 8, 1, 0, 30]
    q["prompt_len"][:] = [0, 30, 5, 0, 8, 1, 0, 29]
    q["entry_bias"][:, 0] = -INF
    q["entry_idx"][:, 0] = 7
    q["bias"][6] = -INF
    for masks in (True, False):
        if not masks:
            q["masks"] = q["mask_of"] = None
        check_forward(ctx, src, z, q)
        check_forward(ctx, src, z, q, over=True)
        check_forward(ctx, src, z, dict(q, bias=None), over=True)
        G = z.clone()
        G[4] = 0.25
        check_backward(ctx, src, z, G, dict(q, bias=None), bias=False)
        check_backward(ctx, src, z, G, dict(q, bias=None), bias=False, over=True)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_rows_with_parameters_out_of_range(ctx, src):
    rows, cols = 16, 5000
    z, q = draw(src, rows, cols, 2), settings(rows, cols, 2, prior=10, entries=3, masks=2, bias=True)
    q["repetition"][:6] = [0.0, -1.0, INF, NAN, 1e-45, 3e38]
    q["frequency"][6:8] = [INF, NAN]
    q["presence"][8:10] = [-INF, NAN]
    q["prior_len"][10:13] = [-1, 11, 5]
    q["prompt_len"][10:13] = [0, 0, 6]
    q["prompt_len"][13] = -1
    q["mask_of"][:] = -1
    q["mask_of"][14:] = [2, -2]
    bad = [r for r in range(rows) if facts(q, r, cols)[2] is None]
    assert bad == [0, 1, 2, 3, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15]
    for over in (False, True):
        check_forward(ctx, src, z, q, over=over)
        check_forward(ctx, src, z, dict(q, bias=None), over=over)
        G = draw(src, rows, cols, 3)
        check_backward(ctx, src, z, G, q, over=over, bias=False)
        check_backward(ctx, src, z, G, q, over=over)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [70, 5000])
def test_lengths_without_a_history(ctx, src, cols):
    """n_prior = 0: rows that say anything but 0 <= prompt_len <= prior_len <= 0 are out of range, with entries, masks, a shared bias and without."""
    import torch
    rows = 7
    lens, prompts = np.int32([0, 5, 0, -1, 0, 3, 0]), np.int32([0, 0, 1, 0, -1, 3, 0])
    z, G = draw(src, rows, cols, 14), draw(src, rows, cols, 15)
    empty = torch.zeros((rows, 0), dtype=torch.int32, device="cuda")
    for n, (entries, masks, bias) in enumerate([(0, 0, False), (3, 0, False), (0, 2, True), (5, 2, True), (0, 0, True)]):
        base = settings(rows, cols, n, 0, entries, masks, bias)
        for given, bad in ((dict(prior_len=lens, prompt_len=prompts), [1, 2, 3, 4, 5]), (dict(prior_len=lens), [1, 3, 5]), (dict(prompt_len=prompts), [2, 4, 5])):
            q = dict(base, **given)
            want, big, word = forward(f64(z), base)
            want[bad] = NAN
            tol = np.nan_to_num(np.where(word, 2.0 ** -50 * big, U * np.abs(want) if bias and src != "f32" else 0.0), nan=0.0, posinf=0.0)
            for near in (dev(q), dict(dev(q), prior=empty)):
                out = torch.full_like(z, 55.0)
                ctx.qsv_adjust(KIND[src], z, out, **near)
                close(src, f64(out), want, tol)
                over = z.clone()
                ctx.qsv_adjust(KIND[src], over, **near)
                close(src, f64(over), want, tol)
                back = {k: v for k, v in near.items() if k not in ("bias", "entry_bias")}
                wgrad, db, ab, de = backward(f64(z), f64(G), base)
                wgrad[bad], de[bad] = NAN, NAN
                db[:] = NAN
                for over in (False, True):
                    for with_bias in (False, True):
                        grad = G.clone() if over else torch.full_like(G, 55.0)
                        b = torch.zeros(cols, device="cuda") if with_bias else None
                        e = torch.zeros(base["entry_idx"].shape, device="cuda") if entries else None
                        ctx.qsv_adjust_grad(KIND[src], grad if over else G, grad=grad, grad_bias=b, grad_entry=e, **back)
                        close(src, f64(grad), wgrad, np.zeros_like(wgrad))
                        assert b is None or bool(b.isnan().all())
                        assert e is None or np.array_equal(f64(e), de, equal_nan=True)


def check_all(ctx, src, z, G, q):
    """Both directions, beside and in place, with and without the shared bias' gradient, without the entries' gradients."""
    import torch
    want, big, word, *_ = forward_all(f64(z), q)
    near = dev(q)
    out = torch.full_like(z, 55.0)
    ctx.qsv_adjust(KIND[src], z, out, **near)
    tol = np.where(word, 2.0 ** -50 * big, U * np.abs(want) if q.get("bias") is not None and src != "f32" else 0.0)
    close(src, f64(out), want, np.nan_to_num(tol, nan=0.0, posinf=0.0))
    want, big, word, *_ = forward_all(f64(z), dict(q, bias=None))
    over = z.clone()
    ctx.qsv_adjust(KIND[src], over, **{k: v for k, v in near.items() if k != "bias"})
    close(src, f64(over), want, np.where(word & ~np.isnan(want), 2.0 ** -50 * big, 0.0))
    back = {k: v for k, v in near.items() if k not in ("bias", "entry_bias")}
    want, db, ab = backward_all(f64(z), f64(G), q)
    for over in (False, True):
        for bias in (False, True):
            grad = G.clone() if over else torch.full_like(G, 55.0)
            b = torch.full((z.shape[1],), 77.0, device="cuda") if bias else None
            ctx.qsv_adjust_grad(KIND[src], grad if over else G, grad=grad, scores=z, grad_bias=b, **back)
            close(src, f64(grad), want, np.where(np.isnan(want), 0.0, 2.0 ** -50 * np.abs(want)))
            # sums of n values in float64, in any order: off by n 2^-53 of the absolute sum at most, and one rounding
            if bias:
                assert ((np.abs(f64(b) - db) <= U * np.abs(db) + len(z) * 2.0 ** -53 * 2.0 * ab + 2.0 ** -149) | (np.isnan(f64(b)) & np.isnan(db))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,prior,entries", [(4225, 70, 12, 0), (5000, 70, 12, 3), (5000, 33, 0, 0), (40000, 70, 12, 3), (40000, 9, 300, 0), (1100003, 3, 3, 1)])
def test_many_rows(ctx, src, rows, cols, prior, entries):
    """Blocks of 33 to 256 rows of the shared bias' sums, the last one short; more workgroups than one dimension of a grid holds."""
    c = ctx
    if qb.qsv_adjust_grad_workspace_bytes(rows, cols) > ctx.ws.numel():
        c = qb.Context(1, 1, ws_bytes=qb.qsv_adjust_grad_workspace_bytes(rows, cols))
    z, G = draw(src, rows, cols, rows), draw(src, rows, cols, rows + 1, sigma=0.2)
    q = settings(rows, cols, rows + cols, prior, entries, 5, True)
    check_all(c, src, z, G, q)
    if prior:
        q["prompt_len"][rows // 2], q["repetition"][rows - 1] = -1, 0.0      # the sums of all columns become NaN
        check_all(c, src, z, G, q)
    if c is not ctx:
        c.close()


@pytest.mark.gpu
def test_sums_of_columns_over_two_dimensions_of_workgroups():
    """4096 rows of more than four million columns: whole numbers, whose sums are exact."""
    import torch
    rows, cols = 4096, (1 << 22) + 517            # 128 blocks of 32 rows, 8194 tiles of 512 columns
    assert rows // 32 * -(-cols // 512) > 1 << 20
    c = qb.Context(1, 1, ws_bytes=qb.qsv_adjust_grad_workspace_bytes(rows, cols))
    k = torch.arange(cols, device="cuda", dtype=torch.int32)
    G = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    want = torch.zeros(cols, dtype=torch.int64, device="cuda")
    for r in range(rows):
        row = (k * (2 * (r % 7) + 1) + r) % 11 - 5
        G[r] = row
        want += row
    words = torch.randint(-2 ** 31, 2 ** 31, (1, (cols + 31) // 32), device="cuda", dtype=torch.int64, generator=torch.Generator("cuda").manual_seed(1)).to(torch.int32)
    allowed = (words.view(-1, 1) >> torch.arange(32, device="cuda", dtype=torch.int32) & 1).flatten()[:cols]
    b = torch.full((cols,), 77.0, device="cuda")
    c.qsv_adjust_grad(KIND["bf16"], G, grad_bias=b, masks=words)
    assert torch.equal(b, (want * allowed).float())
    b.fill_(77.0)
    c.qsv_adjust_grad(KIND["bf16"], G, grad=G, grad_bias=b, masks=words)
    assert torch.equal(b, (want * allowed).float())
    for r in (0, 31, 32, 2049, rows - 1):
        assert torch.equal(G[r].int(), ((k * (2 * (r % 7) + 1) + r) % 11 - 5) * allowed)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(2, 300), (2, 9001)])
def test_longest_histories(ctx, src, rows, cols):
    """2^20 earlier outcomes, all of them one outcome or each at random: counts of 21 bits."""
    n = 1 << 20
    q = settings(rows, cols, 6, prior=n, entries=2, masks=2)
    q["prior"][0], q["prior_len"][0], q["prompt_len"][0] = 7, n, 0
    q["frequency"][:], q["presence"][:], q["repetition"][:] = np.float32(2.0 ** -12), 0.5, 1.25
    q["mask_of"][:] = -1
    z, G = draw(src, rows, cols, 17), draw(src, rows, cols, 18)
    z[0, 7] = 2.0
    check_all(ctx, src, z, G, q)
    q["prompt_len"][0] = n
    check_all(ctx, src, z, G, q)


@pytest.mark.gpu
def test_masks_by_row_and_one_for_all(ctx):
    rows, cols = 6, 777
    z, q = draw("bf16", rows, cols, 5), settings(rows, cols, 5, masks=rows)
    check_forward(ctx, "bf16", z, dict(q, mask_of=None))
    check_forward(ctx, "bf16", z, dict(q, mask_of=None), over=True)
    check_backward(ctx, "bf16", z, z, dict(q, mask_of=None))
    check_forward(ctx, "bf16", z, dict(q, mask_of=None, masks=q["masks"][2:3]))
    check_backward(ctx, "bf16", z, z, dict(q, mask_of=None, masks=q["masks"][2:3]), over=True)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16"])
def test_most_entries_and_all_of_one_outcome(ctx, src):
    rows, cols = 3, 20000
    z, q = draw(src, rows, cols, 6), settings(rows, cols, 6, prior=5, entries=1023)
    q["entry_idx"][0] = 19999
    q["entry_bias"][0] *= np.float32(1e-3)
    q["entry_idx"][1] = 7 + np.arange(1023) % 3
    check_forward(ctx, src, z, q)
    check_forward(ctx, src, z, q, over=True)
    check_backward(ctx, src, z, z, q, bias=False)


@pytest.mark.gpu
def test_addresses_and_strides_beyond_32_bits(ctx):
    import torch
    rows, cols, stride = 3, 2500, (1 << 31) + 5
    z, q = draw("bf16", rows, cols, 7), settings(rows, cols, 7, prior=40, entries=5, masks=2)
    whole = torch.zeros(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    far = whole.as_strided((rows, cols), (stride, 1))
    far.copy_(z)
    want, near = check_forward(ctx, "bf16", z, q), dev(q)
    ctx.qsv_adjust(KIND["bf16"], far, **near)
    assert torch.equal(far.view(torch.int16), want.view(torch.int16))
    assert int(whole.count_nonzero()) <= rows * cols
    far.copy_(z)
    out, grad, near = torch.zeros_like(z), torch.zeros_like(z), {k: v for k, v in near.items() if k != "entry_bias"}
    ctx.qsv_adjust_grad(KIND["bf16"], z, grad=out, scores=z, **near)
    ctx.qsv_adjust_grad(KIND["bf16"], far, grad=grad, scores=far, **near)
    assert torch.equal(out, grad)
    prior = torch.zeros(2 * (1 << 30) + 64, dtype=torch.int32, device="cuda").as_strided((rows, 40), (1 << 30, 1))
    prior.copy_(near["prior"])
    ctx.qsv_adjust_grad(KIND["bf16"], z, grad=grad.zero_(), scores=z, **dict(near, prior=prior))
    assert torch.equal(out, grad)


@pytest.mark.gpu
def test_the_same_bits_every_time(ctx):
    import torch
    rows, cols = 40, 30011
    z, q = draw("f32", rows, cols, 8), settings(rows, cols, 8, prior=2000, entries=100, masks=3, bias=True)
    near, ref = dev(q), None
    back = {k: v for k, v in near.items() if k not in ("bias", "entry_bias")}
    for _ in range(3):
        out, grad, b = torch.zeros_like(z), torch.zeros_like(z), torch.zeros(cols, device="cuda")
        ctx.qsv_adjust(KIND["f32"], z, out, **near)
        ctx.qsv_adjust_grad(KIND["f32"], z, grad=grad, scores=z, grad_bias=b, **back)
        bits = [t.view(torch.int32).clone() for t in (out, grad, b)]
        assert ref is None or all(torch.equal(x, y) for x, y in zip(ref, bits))
        ref = bits


@pytest.mark.gpu
def test_no_rows_and_no_columns_to_change(ctx):
    import torch
    z = torch.zeros((0, 9), device="cuda")
    ctx.qsv_adjust(KIND["f32"], z)
    b = torch.full((9,), 3.0, device="cuda")
    ctx.qsv_adjust_grad(KIND["f32"], z, grad=z, grad_bias=b)
    assert bool((b == 0).all())
    z = draw("f16", 4, 999, 9)
    keep = z.clone()
    ctx.qsv_adjust(KIND["f16"], z)
    ctx.qsv_adjust_grad(KIND["f16"], z, grad=z)
    assert torch.equal(keep, z)


@pytest.mark.gpu
def test_refused_on_the_device(ctx):
    import torch
    z = torch.zeros((4, 64), device="cuda")
    for call in (lambda: ctx.qsv_adjust(KIND["f16"], z), lambda: ctx.qsv_adjust(KIND["f32"], z.cpu()), lambda: ctx.qsv_adjust(KIND["f32"], z, out=z[:, :32]),
                 lambda: ctx.qsv_adjust(KIND["f32"], z[:2], out=z[1:3]), lambda: ctx.qsv_adjust(KIND["f32"], z, bias=torch.zeros(63, device="cuda")),
                 lambda: ctx.qsv_adjust(KIND["f32"], z, entry_idx=torch.zeros((4, 2), dtype=torch.int32, device="cuda")),
                 lambda: ctx.qsv_adjust(KIND["f32"], z, mask_of=torch.zeros(4, dtype=torch.int32, device="cuda")),
                 lambda: ctx.qsv_adjust_grad(KIND["f32"], z, grad=z[:, :32]), lambda: ctx.qsv_adjust_grad(KIND["f32"], z[:2], grad=z[1:3])):
        with pytest.raises(qb.QsvError) as e:
            call()
        assert e.value.status == qb.QSV_ERR_INVALID_ARG
    need = qb.qsv_adjust_grad_workspace_bytes(1 << 20, 262144)
    small = qb.Context(1, 1)
    big = torch.empty((1,), device="cuda")          # never touched: the call is refused
    assert need > small.ws.numel()
    r, b = qb.qsv_adjust_req(), qb.qsv_adjust_grad_req()
    r.kind, r.rows, r.cols, b.grad_out_dev, b.grad_out_stride = KIND["f32"], 1 << 20, 262144, big.data_ptr(), 262144
    b.grad_bias_dev = big.data_ptr()
    assert small.L.qsv_adjust_grad(small.h, ctypes.byref(r), ctypes.byref(b)) == qb.QSV_ERR_WORKSPACE
    assert b"qsv_adjust_grad" in small.L.qsv_last_error(small.h)
    small.close()


@pytest.mark.gpu
def test_serving_step_adjusted_then_sampled(ctx):
    """Scores that have been adjusted in place are drawn from: rows without an outcome and rows out of range give -1."""
    import torch
    rows, cols = 9, 50021
    z, q = draw("bf16", rows, cols, 12), settings(rows, cols, 12, prior=300, entries=12, masks=4)
    q["mask_of"][:] = [-1, 0, 1, 2, 3, 0, 1, 2, -1]           # mask 3 leaves nothing
    q["repetition"][8] = -2.0
    out, u = torch.zeros((rows, 64), dtype=torch.int64, device="cuda"), torch.rand((rows, 64), dtype=torch.float64, device="cuda")
    kept = torch.zeros((rows,), dtype=torch.int32, device="cuda")
    ctx.qsv_adjust(KIND["bf16"], z, **dev(q))
    ctx.qsv_sample(KIND["bf16"], out, u, scores=z, temperature=torch.full((rows,), 3.0, device="cuda"), kept=kept)
    out, kept, v = out.cpu().numpy(), kept.cpu().numpy(), f64(z)
    for r in range(rows):
        a = facts(q, r, cols)[2]
        if a is None or not a.any():
            assert (out[r] == -1).all() and kept[r] == 0
        else:
            assert a[out[r]].all() and kept[r] == np.isfinite(v[r]).sum() and kept[r] == a.sum()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,prior,entries", [(257, 33000, 2100, 1000), (257, 33000, 9000, 5), (3, 4000, 4000, 1023)])
def test_captured_with_large_tables(rows, cols, prior, entries):
    """Parts and rows whose tables take most of a CU's memory, recorded before any eager call has asked for it."""
    import torch
    near = dev(settings(rows, cols, 31, prior, entries, masks=3))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = qb.Context(1, 1)
        z = draw("bf16", rows, cols, 30)
        out, over = torch.zeros_like(z), torch.zeros_like(z)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.qsv_adjust(KIND["bf16"], z, out, **near)
            c.qsv_adjust(KIND["bf16"], over, **near)
        want, want_over = torch.zeros_like(z), z.clone()
        c.qsv_adjust(KIND["bf16"], z, want, **near)
        c.qsv_adjust(KIND["bf16"], want_over, **near)
        for _ in range(3):
            out.fill_(9.0)
            over.copy_(z)
            g.replay()
            stream.synchronize()
            assert torch.equal(out, want) and torch.equal(over, want_over) and torch.equal(out, over)
        c.close()


@pytest.mark.gpu
def test_two_contexts_side_by_side():
    """Calls of two contexts on two streams, under way together, give what each gives alone."""
    import torch
    rows, cols = 300, 20000
    sets = []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            q = dev(settings(rows, cols, 40 + i, prior=400, entries=20, masks=3, bias=True))
            sets.append(dict(c=qb.Context(1, 1), stream=stream, z=draw("f32", rows, cols, 41 + i), q=q,
                             back={k: v for k, v in q.items() if k not in ("bias", "entry_bias")}))
    torch.cuda.synchronize()

    def step(s):
        with torch.cuda.stream(s["stream"]):
            out, grad, b = torch.zeros_like(s["z"]), torch.zeros_like(s["z"]), torch.zeros(cols, device="cuda")
            s["c"].qsv_adjust(KIND["f32"], s["z"], out, **s["q"])
            s["c"].qsv_adjust_grad(KIND["f32"], s["z"], grad=grad, scores=s["z"], grad_bias=b, **s["back"])
        return out, grad, b
    alone = []
    for s in sets:
        alone.append(step(s))
        torch.cuda.synchronize()
    for _ in range(5):
        both = [step(s) for s in sets]
        torch.cuda.synchronize()
        for got, want in zip(both, alone):
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    for s in sets:
        s["c"].close()


@pytest.mark.gpu
def test_captured_steps_replay(ctx):
    """Two graphs on one workspace, replayed in turn with eager work between, give what eager calls give."""
    import torch
    rows, cols = 20, 9001
    q = settings(rows, cols, 13, prior=60, entries=7, masks=3, bias=True)
    near = dev(q)
    back = {k: v for k, v in near.items() if k not in ("bias", "entry_bias")}
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = qb.Context(1, 1)
        sets = []
        for i in range(2):
            z = draw("f16", rows, cols, 20 + i)
            sets.append(dict(z=z, out=torch.zeros_like(z), grad=torch.zeros_like(z), b=torch.zeros(cols, device="cuda"),
                             e=torch.zeros((rows, 7), device="cuda")))

        def step(s):
            c.qsv_adjust(KIND["f16"], s["z"], s["out"], **near)
            c.qsv_adjust_grad(KIND["f16"], s["out"], grad=s["grad"], scores=s["z"], grad_bias=s["b"], grad_entry=s["e"], **back)
        want = []
        for s in sets:
            step(s)
            stream.synchronize()
            want.append({k: s[k].clone() for k in ("out", "grad", "b", "e")})
        graphs = []
        for s in sets:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                step(s)
            graphs.append(g)
        for _ in range(3):
            for s in sets:
                for k in ("out", "grad", "b", "e"):
                    s[k].fill_(9.0)
            for g in graphs:
                g.replay()
            other = torch.randn((64, 64), device="cuda").sum()
            stream.synchronize()
            assert bool(torch.isfinite(other))
            for s, w in zip(sets, want):
                assert all(torch.equal(s[k].nan_to_num(), w[k].nan_to_num()) for k in w)
        c.close()
