"""qsv_distill and qsv_distill_grad against their formulas in 64 bits.

Errors that the kernels may make, for scores whose highest lies d / T above the lowest that counts:
  e_k   the difference, its scale and the product are rounded (3 steps of 2^-24 of an exponent of at most D = min(d / T,
        104) in units of e: beyond, e_k is below 2^-149) and the exponential itself is good to 2 units of 2^-24
        -> relative DELTA_E = (3 D + 2) 2^-24
  s     a thread adds at most N = 16 * 8 values (longer rows: cols / 1024), each partial sum rounded once
        -> relative DELTA_S = DELTA_E + N 2^-24
  loss  Q ln s is off by Q DELTA_S, q by 2^-24 of itself (its logarithms by as much); rounded once to float32
  gradient  g / T (Q e / s - q): the first product by DELTA_E + DELTA_S + 4 2^-24, the second by 2 2^-24, and one rounding to the
        type: half a step, or half its smallest number"""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2602_13140_amd import binding as qb
from paper_2602_13140_amd import workloads as wl
from tests import gpu_util as gu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF, NAN = math.inf, math.nan
U = 2.0 ** -24
RX, RY, RZ = 1, 2, 3
NONE, RING, LADDER = 0, 1, 2


# ---- the formulas ----------------------------------------------------------------------------------------------------
def teacher_q(idx, logits, lse, t, cols):
    """q of every entry and (t_j / T - norm), one row."""
    real = (idx >= 0) & (idx < cols) & (logits > -INF)
    x = logits.astype(np.float64) / t
    if lse is None:
        norm = np.logaddexp.reduce(x[real]) if real.any() else 0.0
    else:
        norm = float(lse)
    with np.errstate(over="ignore"):
        return np.where(real, np.exp(x - norm), 0.0), x - norm


def reference(z, idx, logits, t=1.0, lse=None, grad_loss=None, stats=None):
    """loss [rows], gradient [rows][cols], what bounds their errors, and m and s of float64 scores z."""
    rows, cols = z.shape
    loss, grad, tol_l, tol_g, ms = np.zeros(rows), np.zeros((rows, cols)), np.zeros(rows), np.zeros((rows, cols)), np.zeros((rows, 2))
    for r in range(rows):
        q, lnq = teacher_q(idx[r], logits[r], None if lse is None else lse[r], t, cols)
        g = 1.0 if grad_loss is None else float(grad_loss[r])
        with np.errstate(all="ignore"):
            m = np.nanmax(z[r]) if stats is None else float(stats[r, 0])
            e = np.exp((z[r] - (m if m > -INF else 0.0)) / t)
            s = e.sum() if stats is None else float(stats[r, 1])
        ms[r] = m, s
        if q.sum() == 0:
            continue
        there = z[r][np.isfinite(z[r])]
        D = min((m - there.min()) / t if there.size else 0.0, 104.0)
        n = max(16 * 8, cols / 1024)
        de, ds = (3 * D + 2) * U, ((3 * D + 2) + n) * U
        at = q > 0
        with np.errstate(all="ignore"):
            lnp = (z[r][idx[r][at]] - m) / t - np.log(s)
            lnp[z[r][idx[r][at]] == -INF] = -INF
            loss[r] = (q[at] * (lnq[at] - lnp)).sum()
            p = q.sum() * e / s if s != 0 else np.zeros(cols)
            qs = np.zeros(cols)
            np.add.at(qs, idx[r][at], q[at])
            grad[r] = g / t * (p - qs)
            tol_l[r] = q.sum() * ds + (q[at] * (np.abs(lnq[at]) + np.abs(lnp) + 2)).sum() * U + U * abs(loss[r])
            tol_g[r] = abs(g) / t * (p * (de + ds + 4 * U) + qs * 2 * U)
    return loss, grad, tol_l, tol_g, ms


def test_formulas_against_differences():
    g = np.random.default_rng(0)
    z, idx = g.standard_normal((3, 8)) * 2, np.array([[0, 3, 3], [7, -1, 8], [1, 2, 5]])
    logits = g.standard_normal((3, 3)).astype(np.float32)
    for lse in (None, np.array([2.0, 1.5, 2.5])):
        for t in (1.0, 1.7):
            _, grad, _, _, _ = reference(z, idx, logits, t, lse, grad_loss=np.array([1.0, 2.0, -0.5]))
            for k in range(8):
                h = 1e-5
                zp, zm = z.copy(), z.copy()
                zp[:, k] += h
                zm[:, k] -= h
                d = (reference(zp, idx, logits, t, lse)[0] - reference(zm, idx, logits, t, lse)[0]) / (2 * h)
                assert np.abs(d * [1.0, 2.0, -0.5] - grad[:, k]).max() < 1e-9


# ---- refusals, without a device --------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    lib = str(tmp_path_factory.mktemp("checks") / "checks.so")
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-fsanitize=undefined", "-static-libubsan",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2602_13140_amd", "csrc"),
                           os.path.join(ROOT, "tests", "check_requests.cpp"), "-o", lib])
    L = ctypes.CDLL(lib)
    L.request_distill.restype = ctypes.c_char_p
    L.request_distill.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    return L


def req(**more):
    r = qb.qsv_distill_req()
    r.kind, r.scores_dev, r.rows, r.cols, r.row_stride = qb.QSV_S_BF16, 0x10000, 3, 10, 12
    r.loss_dev, r.grad_dev, r.grad_stride = 0x2000, 0x20000, 10
    for k, v in more.items():
        setattr(r, k, v)
    return r


def teacher(**more):
    t = qb.qsv_teacher(4, 0, 0x4000, 0x5000, None, 1.0)
    for k, v in more.items():
        setattr(t, k, v)
    return t


def test_refusals(checks):
    def say(r, t):
        return checks.request_distill(ctypes.byref(r) if r else None, ctypes.byref(t) if t else None)
    assert say(req(), teacher()) is None
    assert b"req" in say(None, teacher()) and b"teacher" in say(req(), None)
    for kind in (0, qb.QSV_S_PROBS, qb.QSV_S_STATE, 9):
        assert b"kind" in say(req(kind=kind), teacher())
    assert b"rows" in say(req(rows=-1), teacher()) and b"cols" in say(req(cols=0), teacher())
    assert b"row_stride" in say(req(row_stride=9), teacher())
    assert b"scores_dev" in say(req(scores_dev=None), teacher())
    assert b"aligned" in say(req(scores_dev=0x10001), teacher()) and b"aligned" in say(req(grad_dev=0x20001), teacher())
    assert b"grad_stride" in say(req(grad_stride=9), teacher())
    assert b"have_stats" in say(req(have_stats=2), teacher())
    assert b"have_stats" in say(req(have_stats=1), teacher())                               # neither stats
    assert b"have_stats" in say(req(have_stats=1, stats_dev=0x3000), teacher())             # with a loss
    assert say(req(have_stats=1, stats_dev=0x3000, loss_dev=None), teacher()) is None
    assert b"overlap" in say(req(grad_dev=0x10002), teacher())
    assert b"overlap" in say(req(grad_dev=0x10000), teacher())                              # another stride
    assert say(req(grad_dev=0x10000, grad_stride=12), teacher()) is None
    assert say(req(grad_dev=0x10000 + 2 * 12 * 2 + 10 * 2), teacher()) is None              # right behind
    assert b"overlap" in say(req(grad_dev=0x10000 + 2 * 12 * 2 + 10 * 2 - 2), teacher())
    for top in (0, 1025, -3):
        assert b"n_top" in say(req(), teacher(n_top=top))
    assert b"reserved" in say(req(), teacher(reserved=1))
    assert b"top_idx" in say(req(), teacher(top_idx_dev=None)) and b"top_logits" in say(req(), teacher(top_logits_dev=None))
    for t in (0.0, -1.0, NAN, INF):
        assert b"temperature" in say(req(), teacher(temperature=t))
    assert say(req(rows=0, scores_dev=None), None) is None
    assert qb.load().qsv_distill(None, ctypes.byref(req()), ctypes.byref(teacher())) == qb.QSV_ERR_INVALID_ARG
    assert qb.load().qsv_distill_grad(None, None, None, 1, None, None, ctypes.byref(teacher()), None, None, None, None) == qb.QSV_ERR_INVALID_ARG


def test_temperatures_that_32_bits_do_not_take(checks):
    say = lambda t: checks.request_distill(ctypes.byref(req()), ctypes.byref(teacher(temperature=t)))  # noqa: E731
    for t in (1e-310, 1e-39, 1e-31, 2.0 ** -100.5, 2.0 ** 100.5, 1e40, 1e300):
        assert b"temperature" in say(t)
    assert say(2.0 ** -100) is None and say(2.0 ** 100) is None


def test_layouts():
    assert ctypes.sizeof(qb.qsv_teacher) == 40 and ctypes.sizeof(qb.qsv_distill_req) == 80
    assert qb.qsv_distill_workspace_bytes(-1, 5) == 0 == qb.qsv_distill_workspace_bytes(5, 0)
    assert 0 < qb.qsv_distill_workspace_bytes(4096, 131072) and 0 < qb.qsv_distill_workspace_bytes(1, 1 << 30)


def test_tensors_that_the_binding_refuses():
    """By their type, shape, order and device (-1 is the host), as every refusal is raised."""
    import torch
    here = -1
    z = torch.zeros((3, 8))
    assert qb._rows(z, qb.QSV_S_F32, here, "scores") is z and qb._rows(z[:, :5], qb.QSV_S_F32, here, "scores") is not None
    assert qb._rows(torch.zeros((1, 3)).t(), qb.QSV_S_F32, here, "scores") is not None
    for bad, dev in ((None, here), (z[0], here), (z.t(), here), (z[:, ::2], here), (z.half(), here), (z, 0)):
        with pytest.raises(qb.QsvError, match="scores") as e:
            qb._rows(bad, qb.QSV_S_F32, dev, "scores")
        assert e.value.status == qb.QSV_ERR_INVALID_ARG
    with pytest.raises(qb.QsvError, match="kind"):
        qb._rows(z, qb.QSV_S_STATE, here, "scores")
    assert qb._flat(None, "float32", here, "loss", 3) is None
    assert qb._flat(z, "float32", here, "stats", 3, 8) == z.data_ptr() == qb._room(z, "float32", here, "params", 24)
    assert qb._room(z, "float32", here, "params", 20) == z.data_ptr() and qb._room(None, "float32", here, "params", 20) is None
    for bad, dev, count in ((z, here, 25), (z.t(), here, 24), (z.double(), here, 24), (z, 0, 24)):
        with pytest.raises(qb.QsvError, match="params"):
            qb._room(bad, "float32", dev, "params", count)
    for bad, dev, shape in ((z, here, (3, 7)), (z, here, (8, 3)), (z, here, (23,)), (z.t(), here, (8, 3)), (z.double(), here, (3, 8)), (z, 1, (3, 8))):
        with pytest.raises(qb.QsvError, match="stats"):
            qb._flat(bad, "float32", dev, "stats", *shape)
    idx = torch.zeros((3, 2), dtype=torch.int32)
    assert qb._teacher(3, idx, torch.zeros((3, 2)), 1.0, None, here).n_top == 2
    for i, t, lse in ((None, z, None), (idx[0], z, None), (idx.long(), z[:, :2].clone(), None), (idx, z, None), (idx, z[:, :2], None),
                      (idx, z[:, :2].clone(), z[:2, 0].clone())):
        with pytest.raises(qb.QsvError):
            qb._teacher(3, i, t, 1.0, lse, here)
    with pytest.raises(qb.QsvError, match="cuda:0"):
        qb._teacher(3, idx, torch.zeros((3, 2)), 1.0, None, 0)


# ---- on the GPU ------------------------------------------------------------------------------------------------------
KIND = {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16}


def tt(src):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[src]


@pytest.fixture(scope="module")
def ctx():
    c = qb.Context(1, 1)
    yield c
    c.close()


def on_gpu(ctx, src, z, idx, logits, t=1.0, lse=None, grad_loss=None, stats=None, loss=True, grad=True, over=False, pad=0):
    """z: a GPU tensor; the rest numpy.  (loss, gradient, stats) as numpy."""
    import torch
    rows, cols = z.shape
    dev = lambda a, d: None if a is None else torch.as_tensor(np.ascontiguousarray(a)).to(d).cuda()  # noqa: E731
    lo = torch.full((rows,), 77.0, device="cuda") if loss and stats is None else None
    whole = torch.full((rows, cols + pad), 55.0, dtype=tt(src), device="cuda") if grad and not over else None
    gr = z if over else whole[:, :cols] if grad else None
    st = torch.full((rows, 2), 77.0, device="cuda") if stats is None else dev(stats, torch.float32)
    ctx.qsv_distill(KIND[src], z, dev(idx, torch.int32), dev(logits, torch.float32), t, top_lse=dev(lse, torch.float32), loss=lo,
                    stats=st, have_stats=int(stats is not None), grad_loss=dev(grad_loss, torch.float32), grad=gr)
    torch.cuda.synchronize()
    if whole is not None and pad:
        assert bool((whole[:, cols:] == 55.0).all())
    return (lo.cpu().numpy() if lo is not None else None, gr.double().cpu().numpy() if grad else None, st.cpu().numpy())


def compare(src, got, ref):
    import torch
    loss, grad, tol_l, tol_g, ms = ref
    f = torch.finfo(tt(src))
    if got[0] is not None:
        assert np.array_equal(np.isnan(got[0]), np.isnan(loss))
        with np.errstate(invalid="ignore"):
            assert np.all((np.abs(got[0] - loss) <= tol_l) | (got[0] == loss) | np.isnan(loss)), (got[0], loss, tol_l)
    if got[1] is not None:
        assert np.array_equal(np.isnan(got[1]), np.isnan(grad))
        half = np.maximum(f.eps / 2 * np.abs(grad), f.smallest_normal * f.eps / 2)
        with np.errstate(invalid="ignore"):
            ok = np.abs(got[1] - grad) <= (half + tol_g) * (1 + f.eps) + 2.0 ** -126
        assert np.all(ok | np.isnan(grad)), np.nanmax(np.abs(got[1] - grad) / (half + tol_g + 1e-300))


def draw(src, rows, cols, top, seed, sigma=3.0, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((rows, cols + pad), generator=g) * sigma).to(tt(src)).cuda()[:, :cols]
    r = np.random.default_rng(seed)
    idx = np.stack([r.permutation(cols)[:top] if top <= cols else r.integers(0, cols, top) for _ in range(rows)])
    return z, idx, (r.standard_normal((rows, top)) * 2).astype(np.float32)


def f64(z):
    return z.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols,top", [(1, 1), (2, 2), (7, 3), (64, 5), (255, 255), (1000, 1), (1025, 70), (4099, 8), (8193, 300), (16385, 33),
                                      (33001, 64), (70001, 20), (140003, 1024)])
def test_sizes(ctx, src, cols, top):
    rows = 3
    for n, (t, with_lse, pad) in enumerate([(1.0, False, 0), (2.0, True, 3), (0.7, False, 1)]):
        z, idx, logits = draw(src, rows, cols, top, cols + n, pad=pad)
        lse = np.full(rows, 6.0 / t, dtype=np.float32) if with_lse else None
        gl = np.array([1.0, -0.5, 3.0], dtype=np.float32)
        ref = reference(f64(z), idx, logits, t, lse, gl)
        got = on_gpu(ctx, src, z, idx, logits, t, lse, gl, pad=pad)
        compare(src, got, ref)
        assert np.array_equal(got[2][:, 0], ref[4][:, 0].astype(np.float32))
        # the two passes apart, the second from what the first one kept
        back = on_gpu(ctx, src, z, idx, logits, t, lse, gl, stats=got[2])
        compare(src, back, reference(f64(z), idx, logits, t, lse, gl, stats=got[2]))


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(130, 1000), (300, 8200), (129, 33000), (128, 70000), (127, 40000), (1030, 40)])
def test_many_rows(ctx, src, rows, cols):
    z, idx, logits = draw(src, rows, cols, 9, rows)
    idx[1::3, 5:] = -1
    idx[2::7] = cols
    ref = reference(f64(z), idx, logits)
    compare(src, on_gpu(ctx, src, z, idx, logits), ref)
    got = on_gpu(ctx, src, z, idx, logits, grad=False)
    compare(src, got, ref)
    assert np.abs(got[2][:, 1] / ref[4][:, 1] - 1).max() < 1e-4
    assert on_gpu(ctx, src, z, idx, logits, loss=False)[0] is None
    compare(src, on_gpu(ctx, src, z.clone(), idx, logits, over=True), ref)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(12, 500), (12, 40000), (200, 9000)])
def test_masks_and_odd_teachers(ctx, src, rows, cols):
    """Rows that a mask leaves empty or nearly so, the type's lowest value, NaN and infinities, teachers without entries or with the
    same one twice."""
    import torch
    z, idx, logits = draw(src, rows, cols, 6, 5)
    low = torch.finfo(tt(src)).min
    z = z.clone()
    z[0] = -INF
    z[1, 1:] = -INF
    z[2, ::2] = -INF
    z[3, ::2] = low
    z[4] = low
    z[5, 3] = NAN
    z[6, 4] = INF
    idx[0] = [0, 1, 2, 3, 4, 5]
    idx[1] = [0, 0, 0, 0, 0, -1]
    idx[2] = [1, 3, 5, 2, 7, 9]              # one of them masked
    idx[3] = [1, 1, 3, 3, cols - 1, 1]
    idx[7] = -5
    idx[8] = [2, 2, 2, 2, 2, 2]
    logits[9] = -INF
    logits[10, 2:] = -INF
    idx[11] = [2 ** 31 - 1, cols, -2 ** 31, 4, 4, 5]
    ref = reference(f64(z), idx, logits)
    assert np.isinf(ref[0][[0, 2]]).all() and np.isnan(ref[0][[5, 6]]).all() and (ref[0][[7, 9]] == 0).all()
    got = on_gpu(ctx, src, z, idx, logits)
    compare(src, got, ref)
    compare(src, on_gpu(ctx, src, z.clone(), idx, logits, over=True), ref)
    # a row that is not trained on stays at zero whatever its scores are
    z[7, 1] = NAN
    got = on_gpu(ctx, src, z, idx, logits)
    assert got[0][7] == 0 and not got[1][7].any()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(9, 1003), (9, 4099), (9, 9003), (9, 33003), (130, 33003), (130, 132003)])
@pytest.mark.parametrize("what", ["loss", "both"])
def test_infinities_and_nan_wherever_they_stand(ctx, src, rows, cols, what):
    """One +inf or NaN in a row's first value, a middle one, the last ones, which no whole vector has: loss, sum and gradient are
    NaN, the gradient from the kept statistics as well; a row of them that has no entry stays at 0."""
    z, idx, logits = draw(src, rows, cols, 4, 3)
    z = z.clone()
    for r, (k, v) in enumerate([(0, INF), (cols // 2, INF), (cols - 1, INF), (cols - 2, INF), (0, NAN), (cols // 2, NAN), (cols - 1, NAN),
                                (cols - 3, NAN)]):
        z[r, k] = v
    z[8, -3:] = -INF
    idx[:, 0] = 7
    idx[2:4, 1:] = -1
    ref = reference(f64(z), idx, logits)
    assert np.isnan(ref[0][:8]).all() and np.isfinite(ref[0][8:]).all()
    got = on_gpu(ctx, src, z, idx, logits, grad=what == "both")
    compare(src, got, ref)
    assert np.isnan(got[2][:8, 1]).all() and np.isfinite(got[2][8:]).all()
    back = on_gpu(ctx, src, z, idx, logits, stats=got[2])
    assert np.isnan(back[1][:8]).all() and np.isfinite(back[1][8:]).all()
    idx[:8] = -1
    got = on_gpu(ctx, src, z, idx, logits)
    assert not got[0][:8].any() and not got[1][:8].any()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1000), (3, 40000), (200, 9000), (1, 600000)])
def test_loss_of_a_student_near_its_teacher(ctx, rows, cols):
    """The student gives the teacher's entries nearly the teacher's own small probabilities: the terms are q (some 30 less some 30),
    and their difference 2^-10.  What is in 64 bits keeps 2^-50 of each of the two, and the sum s = 1 + sum e is off by the errors
    of e, 2^-16 of e at most at such distances."""
    import torch
    g = np.random.default_rng(cols)
    z = torch.full((rows, cols), -INF, device="cuda")
    z[:, 0] = 0.0
    idx = np.stack([1 + g.permutation(cols - 1)[:5] for _ in range(rows)])
    zt = g.uniform(-40, -25, (rows, 5)).astype(np.float32)
    logits = (zt + np.float32(2.0 ** -10)).astype(np.float32)
    for r in range(rows):
        z[r, torch.as_tensor(idx[r]).cuda()] = torch.as_tensor(zt[r]).cuda()
    lse = np.zeros(rows, dtype=np.float32)
    got = on_gpu(ctx, "f32", z, idx, logits, lse=lse, grad=False)[0]
    q, e = np.exp(logits.astype(np.float64)), np.exp(zt.astype(np.float64))
    want = (q * (logits.astype(np.float64) - zt + np.log1p(e.sum(1, keepdims=True)))).sum(1)
    tol = 2.0 ** -24 * want + (q * 160).sum(1) * 2.0 ** -50 + q.sum(1) * e.sum(1) * 2.0 ** -16
    assert np.all(np.abs(got - want) <= tol), np.abs(got - want) / want


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1000), (3, 40000), (200, 9000)])
def test_an_unlikely_entry_that_the_student_excludes(ctx, rows, cols):
    """q = exp(-110) is less than float32 holds, and not 0."""
    z, idx, logits = draw("f32", rows, cols, 3, 1)
    z = z.clone()
    z[:, 5] = -INF
    idx[:] = [5, 6, 7]
    logits[:] = [-110.0, 0.0, 1.0]
    got = on_gpu(ctx, "f32", z, idx, logits, lse=np.full(rows, 2.0, dtype=np.float32))
    assert np.all(got[0] == INF) and np.isfinite(got[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(2, 40960), (130, 40960), (1, 614400)])
def test_sums_of_parts(rows, cols):
    """s = the ones, one in 2048, and the others at exp(-25) = 2^-36: 2^-25 of the ones together, which 32 bits do not hold beside
    them.  A thread loses the 15 at most that it adds to a one of its own.  The entry's q is 1 / s but for what 64 bits lose, and the
    loss q (ln q - ln p) what the kernel's s is off."""
    import torch
    ctx = qb.Context(1, 1, ws_bytes=max(qb.qsv_workspace_bytes(1, 1), qb.qsv_distill_workspace_bytes(rows, cols)))
    z = torch.full((rows, cols), -25.0, device="cuda")
    z[:, ::2048] = 0.0
    ones = cols // 2048
    s = ones * (1.0 + 2047 * math.exp(-25.0))
    lse = np.float32(math.log(s))
    t = np.float32(float(lse) - math.log(s))
    want = math.exp(float(t) - float(lse)) * ((float(t) - float(lse)) + math.log(s))
    got = on_gpu(ctx, "f32", z, np.zeros((rows, 1)), np.full((rows, 1), t), lse=np.full(rows, lse), grad=False)[0]
    ctx.close()
    assert np.abs(got - want).max() <= 2.0 ** -31 / s, (got[0] * s, want * s)


@pytest.mark.gpu
@pytest.mark.parametrize("src,cols", [("bf16", 4001), ("f16", 30000), ("bf16", 60001), ("bf16", 131072), ("f32", 70003)])
def test_gradients_larger_than_the_caches(ctx, src, cols):
    """Gradients of 384 MiB and more, which are written another way: the same bits as of two calls of half the rows, and of the
    backward pass by itself the same as well."""
    import torch
    size = 4 if src == "f32" else 2
    rows = (384 << 20) // (cols * size) // 2 * 2 + 2
    g = torch.Generator(device="cuda").manual_seed(cols)
    z = (torch.randn((rows, cols), generator=g, device="cuda") * 3).to(tt(src))
    idx = torch.randint(0, cols, (rows, 3), generator=g, device="cuda", dtype=torch.int32)
    logits = torch.randn((rows, 3), generator=g, device="cuda")
    whole, halves = torch.zeros_like(z), torch.zeros_like(z)
    loss, stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, 2), device="cuda")
    ctx.qsv_distill(KIND[src], z, idx, logits, loss=loss, stats=stats, grad=whole)
    h = rows // 2
    for a in (0, h):
        ctx.qsv_distill(KIND[src], z[a:a + h], idx[a:a + h], logits[a:a + h], grad=halves[a:a + h])
    assert torch.equal(whole, halves)
    for a in (0, h):
        ctx.qsv_distill(KIND[src], z[a:a + h], idx[a:a + h], logits[a:a + h], stats=stats[a:a + h], have_stats=1, grad=halves[a:a + h])
    whole.zero_()
    ctx.qsv_distill(KIND[src], z, idx, logits, stats=stats, have_stats=1, grad=whole)
    assert torch.equal(whole, halves)
    at = [0, 1, rows - 1]
    compare(src, (loss[at].cpu().numpy(), f64(whole[at]), None), reference(f64(z[at]), idx[at].cpu().numpy(), logits[at].cpu().numpy()))


@pytest.mark.gpu
def test_gradient_against_differences_of_the_loss(ctx):
    """Central differences of the kernel's own losses: truncation h^2 |f'''| / 6 <= 2^-14 / 6, two losses of up to 8 rounded (2^-21)
    and good to 1e-6 over 2 h = 2^-6."""
    import torch
    z, idx, logits = draw("f32", 2, 11, 4, 3, sigma=1.0)
    grad = on_gpu(ctx, "f32", z, idx, logits)[1]
    h = 2.0 ** -7
    for k in range(11):
        d = torch.zeros_like(z)
        d[:, k] = h
        up, down = (on_gpu(ctx, "f32", z + s * d, idx, logits, grad=False)[0].astype(np.float64) for s in (1, -1))
        assert np.abs((up - down) / (2 * h) - grad[:, k]).max() <= 2.0 ** -14 / 6 + (2 * 2.0 ** -22 + 2e-6) * 2 ** 6


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 524288), (2, 524289), (1, 1048577), (2, 3000001)])
def test_long_rows(src, rows, cols):
    import torch
    ctx = qb.Context(1, 1, ws_bytes=max(qb.qsv_workspace_bytes(1, 1), qb.qsv_distill_workspace_bytes(rows, cols)))
    z, idx, logits = draw(src, rows, cols, 9, cols)
    z[:, 5::7] = -INF
    z[0, cols // 2:] = -INF
    idx[:, 0] = cols - 1
    idx[:, 1] = cols - 2
    for r in range(rows):
        z[r, torch.as_tensor(idx[r]).cuda()] = 0.25          # (no entry at a masked score)
    ref = reference(f64(z), idx, logits, 0.8)
    got = on_gpu(ctx, src, z, idx, logits, 0.8)
    compare(src, got, ref)
    compare(src, on_gpu(ctx, src, z, idx, logits, 0.8, grad=False), ref)
    compare(src, on_gpu(ctx, src, z, idx, logits, 0.8, stats=got[2]), ref)
    ctx.close()


@pytest.mark.gpu
def test_the_longest_row():
    """2^30 scores, the gradient over them: few are not masked, and only there anything is written but 0."""
    import torch
    cols = 1 << 30
    c = qb.Context(1, 1, ws_bytes=max(qb.qsv_workspace_bytes(1, 1), qb.qsv_distill_workspace_bytes(1, cols)))
    z = torch.full((1, cols), -INF, device="cuda")
    at = [0, 1, cols // 2 - 1, cols - 2, cols - 1]
    v = np.array([0.5, -1.0, 2.0, 1.5, -0.25])
    for k, x in zip(at, v):
        z[0, k] = float(x)
    idx, logits = np.array([[cols - 1, cols // 2 - 1]]), np.array([[0.0, 1.0]], dtype=np.float32)
    loss, _, stats = on_gpu(c, "f32", z, idx, logits, grad=False)
    p = np.exp(v - 2.0)
    q = np.exp([0.0, 1.0]) / (1 + math.e)
    want = (q * (np.log(q) - (v[[4, 2]] - 2.0 - math.log(p.sum())))).sum()
    assert abs(loss[0] - want) <= 1e-6 and abs(stats[0, 1] - p.sum()) <= 1e-6
    lo = torch.zeros(1, device="cuda")
    c.qsv_distill(qb.QSV_S_F32, z, torch.as_tensor(idx).int().cuda(), torch.as_tensor(logits).cuda(), loss=lo, grad=z)
    torch.cuda.synchronize()
    g = p / p.sum()
    g[4] -= q[0]
    g[2] -= q[1]
    assert abs(lo.item() - want) <= 1e-6
    assert np.abs(np.array([z[0, k].item() for k in at]) - g).max() <= 1e-6
    assert int(torch.count_nonzero(z).item()) == 5
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(3, 40), (3, 40000), (200, 9000)])
def test_lowest_and_highest_temperature(ctx, src, rows, cols):
    """At 2^100 all that is not masked is as likely; at 2^-100 the highest is certain, and the others are too far for any loss
    but the distance over T."""
    z, idx, logits = draw(src, rows, cols, 1, 5)
    z[:, 1] = -INF
    z[:, 2] = 30.0
    idx[:] = 2
    loss, grad, stats = on_gpu(ctx, src, z, idx, logits, 2.0 ** 100)
    assert np.abs(loss - math.log(cols - 1)).max() <= 1e-5 and np.abs(stats[:, 1] - (cols - 1)).max() <= 1e-5 * cols
    assert np.all(np.isfinite(grad)) and np.abs(grad).max() <= 1e-30
    loss, grad, stats = on_gpu(ctx, src, z, idx, logits, 2.0 ** -100)
    assert np.all(loss == 0) and np.all(grad == 0) and np.all(stats[:, 1] == 1)
    idx[:] = 3
    loss, _, _ = on_gpu(ctx, src, z, idx, logits, 2.0 ** -100, grad=False)
    far = (30.0 - f64(z)[:, 3]) * 2.0 ** 100
    assert np.abs(loss - far).max() <= 1e-6 * far.max()


@pytest.mark.gpu
def test_the_backward_pass_needs_no_workspace():
    """Rows whose forward pass needs more than the context's workspace; the gradient from kept statistics, over the scores."""
    import torch
    c = qb.Context(1, 1)
    rows, cols = 127, (1 << 28) + (1 << 25) + 3
    assert qb.qsv_distill_workspace_bytes(rows, cols) > qb.qsv_workspace_bytes(1, 1)
    if torch.cuda.mem_get_info()[0] < rows * cols * 2 + (8 << 30):
        pytest.skip("the device has not enough free memory")
    z = torch.full((rows, cols), -INF, dtype=torch.bfloat16, device="cuda")
    z[:, 5], z[:, cols - 1] = 1.0, 2.0
    idx = torch.tensor([[cols - 1, 5]], dtype=torch.int32, device="cuda").repeat(rows, 1)
    logits = torch.tensor([[0.0, 1.0]], device="cuda").repeat(rows, 1)
    stats = torch.tensor([[2.0, 1 + math.exp(-1)]], device="cuda").repeat(rows, 1)
    loss = torch.full((rows,), -7.0, device="cuda")
    with pytest.raises(qb.QsvError) as refused:
        c.qsv_distill(qb.QSV_S_BF16, z, idx, logits, loss=loss)
    assert refused.value.status == qb.QSV_ERR_WORKSPACE
    c.qsv_distill(qb.QSV_S_BF16, z, idx, logits, stats=stats, have_stats=1, grad=z)
    torch.cuda.synchronize()
    p, q = 1 / (1 + math.exp(-1)), 1 / (1 + math.e)
    for r in (0, 64, rows - 1):
        assert int(torch.count_nonzero(z[r]).item()) == 2
        assert abs(z[r, cols - 1].item() - (p - q)) <= 2.0 ** -8 and abs(z[r, 5].item() - (q - p)) <= 2.0 ** -8
    assert bool((loss == -7).all())
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_a_row_does_not_depend_on_its_alignment(ctx, src):
    import torch
    g = torch.Generator().manual_seed(5)
    flat = (torch.randn(300000, generator=g) * 3).to(tt(src)).cuda()
    for rows, cols in ((2, 5), (3, 1001), (2, 60001), (200, 900)):
        for off in (0, 1, 3):
            z = torch.as_strided(flat, (rows, cols), (cols + 7, 1), off)
            idx, logits = np.tile([0, cols - 1, 2], (rows, 1)), np.ones((rows, 3), dtype=np.float32)
            compare(src, on_gpu(ctx, src, z, idx, logits, pad=off), reference(f64(z), idx, logits))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(4, 60000), (200, 3001)])
def test_replays_of_a_captured_step(rows, cols):
    import torch
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = qb.Context(1, 1)
        z, idx, logits = draw("bf16", rows, cols, 5, 1)
        z = z.contiguous()
        ti, tl = torch.as_tensor(idx).int().cuda(), torch.as_tensor(logits).cuda()
        loss, grad = torch.zeros(rows, device="cuda"), torch.zeros_like(z)
        call = lambda: c.qsv_distill(qb.QSV_S_BF16, z, ti, tl, loss=loss, grad=grad)  # noqa: E731
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for i in range(4):
            z.copy_(torch.randn((rows, cols), generator=torch.Generator().manual_seed(i)) * (i + 1))
            loss.fill_(-7)
            grad.fill_(-7)
            graph.replay()
            stream.synchronize()
            a = loss.cpu().numpy(), f64(grad), None
            compare("bf16", a, reference(f64(z), idx, logits))
            grad.fill_(-7)
            call()
            stream.synchronize()
            assert np.array_equal(f64(grad), a[1])
        c.close()


@pytest.mark.gpu
def test_refused_calls_leave_their_outputs(ctx):
    import torch
    whole, idx, logits = draw("f32", 3, 21, 2, 1)
    z, idx = whole[:, :20], idx % 20
    loss, ti, tl = torch.full((3,), -7.0, device="cuda"), torch.as_tensor(idx).int().cuda(), torch.as_tensor(logits).cuda()
    for more in (dict(temperature=0.0), dict(have_stats=1), dict(grad=whole[:, 1:])):
        with pytest.raises(qb.QsvError):
            ctx.qsv_distill(qb.QSV_S_F32, z, ti, tl, loss=loss, **more)
    torch.cuda.synchronize()
    assert bool((loss == -7).all())


@pytest.mark.gpu
def test_tensors_refused_before_anything_runs(ctx):
    """Host tensors, another type, too few results: refused with asserts left out as well, and nothing is written."""
    import torch
    z, idx, logits = torch.zeros((3, 20), device="cuda"), torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda")
    loss = torch.full((3,), -7.0, device="cuda")
    for scores, more in ((z.cpu(), {}), (z.half(), {}), (z, dict(loss=loss[:2])), (z, dict(grad=z[:, :19])), (z, dict(stats=loss)),
                         (z, dict(grad_loss=loss.cpu())), (z, dict(top_lse=loss.double()))):
        with pytest.raises(qb.QsvError):
            ctx.qsv_distill(qb.QSV_S_F32, scores, idx, logits, **dict(dict(loss=loss), **more))
    out, u = torch.full((3, 1), -7, dtype=torch.int64, device="cuda"), torch.zeros((3, 1), dtype=torch.float64, device="cuda")
    for more in (dict(scores=z.cpu()), dict(scores=None), dict(uniforms=u.cpu()), dict(uniforms=u.float()), dict(top_k=loss), dict(out=out[:2]),
                 dict(temperature=loss[:2]), dict(kind=qb.QSV_S_STATE)):
        with pytest.raises(qb.QsvError):
            ctx.qsv_sample(**dict(dict(kind=qb.QSV_S_F32, out=out, uniforms=u, scores=z), **more))
    c = qb.Context(2, 3)
    circ = qb.make_circuit(1, [RY], NONE, 1)
    good = dict(x=torch.ones((3, 4), device="cuda"), params=torch.zeros(4, device="cuda"), feats=torch.zeros((3, 2), device="cuda"), loss=loss,
                grad=torch.full((3, 4), -7.0, device="cuda"))
    for k, bad in (("x", good["x"].cpu()), ("x", good["x"].t()), ("params", good["params"][:3]), ("feats", good["feats"][:2]), ("feats", good["feats"].cpu()),
                   ("loss", loss[:2]), ("grad", good["grad"][:, :3]), ("grad", good["grad"][:2]), ("mean_grad", loss), ("mean_loss", loss[:0])):
        with pytest.raises(qb.QsvError):
            c.qsv_distill_grad(circ, top_idx=idx, top_logits=logits, **dict(good, **{k: bad}))
    torch.cuda.synchronize()
    assert bool((loss == -7).all()) and bool((out == -7).all()) and bool((good["grad"] == -7).all())
    c.qsv_distill_grad(circ, top_idx=idx, top_logits=logits, **good)
    torch.cuda.synchronize()
    assert bool((loss != -7).all())
    c.close()


# ---- a circuit's own outcomes ----------------------------------------------------------------------------------------
def circuit_reference(oracle, spec, n, x, params, feats, idx, logits, t, lse):
    """Loss and gradient by the chain rule over the probabilities, whose derivatives are their shifts: dp/dangle =
    (p(angle + pi/2) - p(angle - pi/2)) / 2, times the feature for a re-uploading weight."""
    oc = oracle.make_circuit(spec.n_layers, list(spec.rot), spec.entangler, spec.reupload)

    def probs(b, pr):
        s, _ = oracle.amp_encode(x[b:b + 1], n)
        oracle.apply_layers(s, oc, pr, None if feats is None else feats[b:b + 1])
        return (np.abs(s) ** 2).reshape(-1)
    B, P = x.shape[0], len(params)
    loss, grad, tol = np.zeros(B), np.zeros((B, P)), np.zeros(B)
    slots = spec.slots()
    for b in range(B):
        p = probs(b, params)
        q, lnq = teacher_q(idx[b], logits[b], None if lse is None else lse[b], t, 1 << n)
        at = q > 0
        k = idx[b][at]
        loss[b] = (q[at] * (lnq[at] - np.log(p[k]))).sum()
        tol[b] = 2 * (q[at] * 3e-7 * (0.5 / p[k] + 1 / np.sqrt(p[k]))).sum() + 1e-6
        for i in range(P):
            weight = spec.reupload and (i // n) % slots == 0
            f = float(feats[b, i % n]) if weight else 1.0
            d = []
            for sign in (1, -1):
                pr = params.astype(np.float64).copy()
                pr[i] += sign * math.pi / 2 / f
                d.append(probs(b, pr))
            grad[b, i] = -(q[at] / p[k] * f * (d[0][k] - d[1][k]) / 2).sum()
    return loss, grad, tol


def case(n, B, L, rot, ent, reup, seed, top):
    spec = wl.CircuitSpec(L, tuple(rot), ent, reup)
    g = np.random.default_rng(seed)
    params = wl.draw_params(spec, n, seed)
    x = g.standard_normal((B, 1 << n)).astype(np.float32)
    feats = (g.standard_normal((B, n)) + np.sign(g.standard_normal((B, n)))).astype(np.float32) if reup else None
    return spec, g, params, x, feats, (g.standard_normal((B, top))).astype(np.float32)


CIRCUITS = [(1, 2, 2, (RY, RZ), NONE, 0), (2, 3, 1, (RX,), RING, 0), (4, 3, 2, (RY, RZ), RING, 1), (6, 2, 2, (RX, RY, RZ), LADDER, 0),
            (10, 2, 2, (RY, RZ), RING, 0), (11, 2, 1, (RY, RZ), LADDER, 1), (13, 2, 2, (RY,), RING, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,B,L,rot,ent,reup", CIRCUITS)
@pytest.mark.parametrize("mode", ["default", "naive", "chunk1", "whole"])
def test_circuit(oracle, n, B, L, rot, ent, reup, mode):
    import torch
    top = min(5, 1 << n)
    spec, g, params, x, feats, logits = case(n, B, L, rot, ent, reup, 50 + n, top)
    oc = oracle.make_circuit(L, list(rot), ent, reup)
    s, _ = oracle.amp_encode(x, n)
    oracle.apply_layers(s, oc, params, feats)
    p = np.abs(s) ** 2
    likely = np.argsort(-p, axis=1)[:, :max(top, (1 << n) // 4)]          # outcomes of a quarter of the state, none of them rare
    idx = np.stack([g.permutation(likely[b])[:top] for b in range(B)])
    if top >= 4:
        idx[0, 1] = idx[0, 0]
        idx[1, 2] = -1
    lse = np.full(B, 2.5, dtype=np.float32) if n % 2 else None
    ref = circuit_reference(oracle, spec, n, x, params, feats, idx, logits, 1.3, lse)
    c = gu.make_ctx(n, B, naive=int(mode == "naive"))
    if mode == "chunk1":
        c.qsv_set_option("grad_chunk_rows", 1)
    if mode == "whole":
        c.qsv_set_option("grad_layered", 0)
    c.state.fill_(3.0)
    P = len(params)
    loss, grad = torch.zeros(B, device="cuda"), torch.zeros((B, P), device="cuda")
    ml, mg = torch.zeros(1, device="cuda"), torch.zeros(P, device="cuda")
    c.qsv_distill_grad(qb.circuit_from_spec(spec), gu.dev(x), gu.dev(params), gu.dev(feats) if reup else None,
                       gu.dev(idx.astype(np.int32)), gu.dev(logits), loss, grad, ml, mg, temperature=1.3,
                       top_lse=None if lse is None else gu.dev(lse))
    torch.cuda.synchronize()
    gl, gg = loss.cpu().numpy(), grad.cpu().numpy()
    assert np.all(np.abs(gl - ref[0]) <= ref[2] + 1e-5)
    assert np.all(np.abs(gg - ref[1]).max(axis=1) <= ref[2] + 1e-5)
    assert np.linalg.norm(gg - ref[1]) <= 1e-3 * np.linalg.norm(ref[1])
    assert abs(ml.item() - gl.mean()) <= 1e-5 * max(1, abs(gl.mean())) and np.abs(mg.cpu().numpy() - gg.mean(0)).max() <= 1e-5 * max(1, np.abs(gg).max())
    assert bool((c.state == 3.0).all())
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n,B,L,opts", [(14, 4, 40, {}), (13, 12, 64, {"grad_chunk_rows": 5}), (12, 12, 64, {}), (15, 12, 64, {}),
                                        (16, 3, 40, {"tile_log2": 10})])
@pytest.mark.parametrize("reup", [0, 1])
def test_circuit_losses_without_the_rounding_of_their_scalars(oracle, n, B, L, opts, reup):
    """Rotations of 10 qubits about one axis, no entangler, no amplitude where another qubit reads 1, and a teacher that gives each of
    the 1024 outcomes its own probability: the loss is what the state's length is off.  A rotation rounds an amplitude 1.5
    times (three multiply-adds for two), up or down as it comes, by 5e-8 of 2^-5 at one standard deviation; so the length is off
    by 2 * 5e-8 sqrt(10 L) 2^-5, and four times that is the tolerance.  The scalar that a group of unitaries shares makes all
    amplitudes longer or shorter, by 3e-8 a group, of which there are dozens."""
    torch = gu.torch_cuda()
    spec = wl.CircuitSpec(L, () if reup else (RY,), NONE, reup)
    circ, P = qb.circuit_from_spec(spec), spec.num_params(n)
    g = np.random.default_rng(n)
    still = g.permutation(n)[:n - 10]
    live = np.flatnonzero((np.arange(1 << n) & sum(1 << int(q) for q in still)) == 0)
    x = np.zeros((B, 1 << n), dtype=np.float32)
    x[:, live] = g.standard_normal((B, 1024))
    f = g.standard_normal((B, n)).astype(np.float32)
    p = (g.random((L, n)) * 6.0).astype(np.float32)
    p[:, still] = 0.0
    p = p.reshape(-1)
    s, _ = oracle.amp_encode(x, n)
    oracle.apply_layers(s, oracle.make_circuit(L, list(spec.rot), NONE, reup), p, f if reup else None)
    top = (np.abs(s) ** 2).reshape(B, -1)[:, live]
    logits = np.log(top).astype(np.float32)
    want = (np.exp(logits.astype(np.float64)) * (logits - np.log(top))).sum(1)
    c = gu.make_ctx(n, B, ws_bytes=qb.qsv_grad_workspace_bytes(n, B, circ))
    for k, v in opts.items():
        c.qsv_set_option(k, v)
    loss, grad = torch.zeros(B, device="cuda"), torch.zeros((B, P), device="cuda")
    c.qsv_distill_grad(circ, gu.dev(x), gu.dev(p), gu.dev(f) if reup else None, gu.dev(np.tile(live, (B, 1)).astype(np.int32)), gu.dev(logits),
                       loss, grad, top_lse=torch.zeros(B, device="cuda"))
    torch.cuda.synchronize()
    c.close()
    err = loss.cpu().numpy() - want
    assert np.abs(err).max() <= 4 * 2 * 5e-8 * math.sqrt(10 * L) * 2.0 ** -5, err


@pytest.mark.gpu
@pytest.mark.parametrize("n,B,L,rot,ent,reup,opts", [
    (13, 5, 3, (RY, RZ), RING, 0, {"tile_log2": 10}),                                          # deferred CNOTs: passes with an index map
    (13, 5, 3, (RY, RZ), RING, 0, {"tile_log2": 10, "split_streams": 1, "grad_chunk_rows": 2}),  # three chunks on two streams
    (12, 6, 2, (RX, RY), LADDER, 1, {"split_streams": 1}),                                     # halves on two streams, tables of their own
    (14, 3, 4, (RY, RX), RING, 1, {"tile_log2": 11, "split_streams": 1, "grad_chunk_rows": 1}),
    (11, 4, 2, (RY, RZ), RING, 0, {"tile_log2": 10, "defer_cnots": 0}),
    (10, 2100, 1, (RY,), RING, 0, {}),                                                         # 10 qubits in whole passes
])
def test_circuit_in_whole_passes_and_layer_by_layer(oracle, n, B, L, rot, ent, reup, opts):
    """The loss and gradient of every sample the same both ways, and against the formulas for the first sample, one in the middle
    and the last one."""
    torch = gu.torch_cuda()
    spec, g, params, x, feats, logits = case(n, B, L, rot, ent, reup, 90 + n, 5)
    oc = oracle.make_circuit(L, list(rot), ent, reup)
    s, _ = oracle.amp_encode(x, n)
    oracle.apply_layers(s, oc, params, feats)
    p = np.abs(s) ** 2
    likely = np.argsort(-p, axis=1)[:, :(1 << n) // 4]
    idx = np.stack([g.permutation(likely[b])[:5] for b in range(B)])
    idx[B - 1, 2] = idx[B - 1, 1]
    idx[0, 4] = -1
    circ, P = qb.circuit_from_spec(spec), len(params)
    got = []
    for o in (opts, {"naive": 1}):
        c = gu.make_ctx(n, B, ws_bytes=qb.qsv_grad_workspace_bytes(n, B, circ))
        for k, v in o.items():
            c.qsv_set_option(k, v)
        loss, grad = torch.zeros(B, device="cuda"), torch.zeros((B, P), device="cuda")
        for _ in range(2):
            loss.fill_(7.0), grad.fill_(7.0)
            c.qsv_distill_grad(circ, gu.dev(x), gu.dev(params), gu.dev(feats) if reup else None, gu.dev(idx.astype(np.int32)),
                               gu.dev(logits), loss, grad, temperature=1.3)
            torch.cuda.synchronize()
            got.append((loss.cpu().numpy(), grad.cpu().numpy()))
        c.close()
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
    at = sorted({0, B // 2, B - 1})
    ref = circuit_reference(oracle, spec, n, x[at], params, None if feats is None else feats[at], idx[at], logits[at], 1.3, None)
    for l, gr in got:
        assert np.all(np.abs(l[at] - ref[0]) <= ref[2] + 1e-5)
        assert np.all(np.abs(gr[at] - ref[1]).max(axis=1) <= ref[2] + 1e-5)
    # (each way is off by the tolerance of the formulas' test at most)
    pk = np.take_along_axis(p.reshape(B, -1), idx.clip(0), 1)
    tol = 2 * (2 * 3e-7 * (0.5 / pk + 1 / np.sqrt(pk)).max(1) + 1e-6 + 1e-5)
    assert np.all(np.abs(got[0][0] - got[2][0]) <= tol) and np.all(np.abs(got[0][1] - got[2][1]).max(1) <= tol)


def test_the_circuits_workspace():
    c = qb.make_circuit(6, [RY, RZ], RING)
    for n, B in ((4, 3), (22, 2)):
        more = qb.qsv_distill_grad_workspace_bytes(n, B, c) - qb.qsv_grad_workspace_bytes(n, B, c)
        assert B * (8 << n) <= more < B * (8 << n) + 256
    assert qb.qsv_distill_grad_workspace_bytes(0, 1, c) == 0 == qb.qsv_distill_grad_workspace_bytes(4, 1, qb.make_circuit(1, [9], 1))


@pytest.mark.gpu
@pytest.mark.parametrize("n,B,L,ent", [(22, 2, 6, RING), (24, 2, 3, LADDER), (22, 4, 2, RING)])
def test_circuit_workspace_for_whole_passes(n, B, L, ent):
    """Circuits with as many passes as qsv_grad_workspace_bytes has states for: with one more a sample the call goes the way that it
    goes with many more, bit by bit."""
    import torch
    spec = wl.CircuitSpec(L, (RY, RZ), ent, 0)
    circ, P = qb.circuit_from_spec(spec), spec.num_params(n)
    g = torch.Generator(device="cuda").manual_seed(n)
    x, p = torch.randn((B, 1 << n), device="cuda", generator=g), torch.rand(P, device="cuda", generator=g)
    idx = torch.randint(0, 1 << n, (B, 7), device="cuda", generator=g, dtype=torch.int32)
    logits = torch.randn((B, 7), device="cuda", generator=g)
    ws, got = qb.qsv_distill_grad_workspace_bytes(n, B, circ), []
    for size in (ws, ws + (2 << 30)):
        c = gu.make_ctx(n, B, ws_bytes=size)
        loss, grad = torch.full((B,), 7.0, device="cuda"), torch.full((B, P), 7.0, device="cuda")
        c.qsv_distill_grad(circ, x, p, None, idx, logits, loss, grad)
        torch.cuda.synchronize()
        got.append((loss.clone(), grad.clone()))
        c.close()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(torch.isfinite(got[0][1]).all())


@pytest.mark.gpu
def test_circuit_special_rows():
    """A teacher without entries, an outcome of amplitude 0, no layers; refusals that need a context."""
    import torch
    c = qb.Context(3, 3)
    circ = qb.make_circuit(1, [RZ], NONE)                 # phases only: the outcomes stay as encoded
    x = torch.zeros((3, 8), device="cuda")
    x[:, 0] = 1.0
    x[:, 1] = 1.0
    pr = torch.full((3,), 0.3, device="cuda")
    idx = torch.tensor([[0, 1], [-1, 9], [0, 5]], dtype=torch.int32, device="cuda")
    logits = torch.zeros((3, 2), device="cuda")
    loss, grad = torch.full((3,), 7.0, device="cuda"), torch.full((3, 3), 7.0, device="cuda")
    c.qsv_distill_grad(circ, x, pr, None, idx, logits, loss, grad)
    torch.cuda.synchronize()
    assert abs(loss[0].item()) < 1e-6 and loss[1].item() == 0 and loss[2].item() == INF
    assert bool(torch.isfinite(grad).all()) and grad.abs().max().item() < 1e-6
    none = qb.make_circuit(0, [RZ], NONE)
    loss.fill_(7.0)
    c.qsv_distill_grad(none, x, None, None, idx, logits, loss, None)
    torch.cuda.synchronize()
    assert abs(loss[0].item()) < 1e-6 and loss[1].item() == 0 and loss[2].item() == INF
    with pytest.raises(qb.QsvError, match="temperature"):
        c.qsv_distill_grad(circ, x, pr, None, idx, logits, loss, grad, temperature=0.0)
    with pytest.raises(qb.QsvError, match="teacher"):
        c._check(c.L.qsv_distill_grad(c.h, ctypes.byref(circ), x.data_ptr(), 8, pr.data_ptr(), None, None, loss.data_ptr(), grad.data_ptr(), None, None))
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 11])
def test_circuit_amplitudes_below_the_normal_range(n):
    """An entry at an outcome whose amplitude's inverse 32 bits do not hold: the gradient is that of the other entries."""
    import torch
    c = qb.Context(n, 2)
    circ = qb.make_circuit(1, [RY], NONE)
    x = torch.zeros((2, 1 << n), device="cuda")
    x[:, 0], x[:, 1], x[:, 6] = 0.8, 0.6, 1e-41
    pr = torch.zeros(n, device="cuda")
    logits = torch.zeros((2, 2), device="cuda")
    lse = torch.full((2,), 0.5, device="cuda")
    got = []
    for second in (6, -1):
        idx = torch.tensor([[0, second], [1, second]], dtype=torch.int32, device="cuda")
        loss, grad = torch.full((2,), 7.0, device="cuda"), torch.full((2, n), 7.0, device="cuda")
        c.qsv_distill_grad(circ, x, pr, None, idx, logits, loss, grad, top_lse=lse)
        torch.cuda.synchronize()
        assert not bool(torch.isnan(loss).any())
        got.append(grad.cpu())
    assert bool(torch.isfinite(got[0]).all()) and torch.equal(got[0], got[1]) and got[0].abs().max().item() > 0.1
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n,B,ent,opts", [(5, 3, RING, {}), (10, 1100, RING, {}), (13, 6, RING, {"tile_log2": 10}), (12, 4, LADDER, {"split_streams": 1})])
def test_replays_of_a_captured_circuit_step(n, B, ent, opts):
    """Loss, gradient and an optimiser's step in a graph: layer by layer, in whole passes, with index maps, on two streams.  New inputs,
    parameters and teachers between the replays, each against the same call made eagerly, bit by bit."""
    import torch
    spec = wl.CircuitSpec(2, (RY, RZ), ent, 0)
    circ, P = qb.circuit_from_spec(spec), spec.num_params(n)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = gu.make_ctx(n, B, ws_bytes=qb.qsv_distill_grad_workspace_bytes(n, B, circ))
        for k, v in opts.items():
            c.qsv_set_option(k, v)
        x, p = torch.ones((B, 1 << n), device="cuda"), torch.zeros(P, device="cuda")
        idx, logits = torch.zeros((B, 4), dtype=torch.int32, device="cuda"), torch.zeros((B, 4), device="cuda")
        loss, grad, ml, mg = (torch.zeros(s, device="cuda") for s in ((B,), (B, P), (1,), (P,)))

        def call():
            c.qsv_distill_grad(circ, x, p, None, idx, logits, loss, grad, ml, mg)
            c.qsv_sgd_step(p, mg, 0.05)
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        g = torch.Generator(device="cuda").manual_seed(n)
        for i in range(4):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
            start = torch.rand(P, device="cuda", generator=g) * 3
            idx.copy_(torch.randint(-1, 1 << n, idx.shape, device="cuda", generator=g))
            logits.copy_(torch.randn(logits.shape, device="cuda", generator=g))
            got = []
            for go in (graph.replay, call):
                p.copy_(start)
                for t in (loss, grad, ml, mg):
                    t.fill_(-7.0)
                go()
                stream.synchronize()
                got.append([t.clone() for t in (loss, grad, ml, mg, p)])
            assert all(torch.equal(a, b) for a, b in zip(*got)) and bool(torch.isfinite(got[0][0]).all()) and not torch.equal(got[0][4], start)
        c.close()


@pytest.mark.gpu
def test_contexts_side_by_side():
    """Two contexts, a stream each, whose calls run at once: rows in parts, long rows, many shots; the results are those of calls alone."""
    import torch
    from tests.test_sample import reference as sampled, same, values_of
    g = torch.Generator().manual_seed(2)
    u = torch.rand((3, 40), generator=g, dtype=torch.float64)
    sides = []
    for i in range(2):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            z, idx, logits = draw("f32", 3, 300001 + i, 6, i)
            z = z.contiguous()
            sides.append(dict(st=st, c=qb.Context(1, 1), z=z, idx=idx, logits=logits, ti=torch.as_tensor(idx).int().cuda(), tl=torch.as_tensor(logits).cuda(),
                              loss=torch.zeros(3, device="cuda"), grad=torch.zeros_like(z), u=u.cuda(), out=torch.zeros((3, 40), dtype=torch.int64, device="cuda"),
                              kept=torch.zeros(3, dtype=torch.int32, device="cuda"), p=torch.full((3,), 0.9, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for s in sides:
            with torch.cuda.stream(s["st"]):
                s["c"].qsv_distill(qb.QSV_S_F32, s["z"], s["ti"], s["tl"], loss=s["loss"], grad=s["grad"])
                s["c"].qsv_sample(qb.QSV_S_F32, s["out"], s["u"], scores=s["z"], kept=s["kept"], top_p=s["p"])
    torch.cuda.synchronize()
    for s in sides:
        compare("f32", (s["loss"].cpu().numpy(), f64(s["grad"]), None), reference(f64(s["z"]), s["idx"], s["logits"]))
        same((s["out"].cpu().numpy(), None, s["kept"].cpu().numpy()), sampled(values_of("f32", s["z"]), True, u.numpy(), dict(top_p=[0.9] * 3)))
        s["c"].close()


@pytest.mark.gpu
def test_training_towards_a_teacher_and_answers(oracle):
    """Steps of a circuit towards a teacher's likeliest outcomes, then answers drawn from what it learnt: every step's gradient and
    the drawn outcomes against the references."""
    import torch
    from tests.test_sample import reference as sampled, values_of
    n, B, top = 5, 2, 4
    spec, g, params, x, _, logits = case(n, B, 2, (RY, RZ), RING, 0, 8, top)
    idx = np.stack([g.permutation(1 << n)[:top] for _ in range(B)])
    c, circ, P = qb.Context(n, B), qb.circuit_from_spec(spec), len(params)
    xd, pd = gu.dev(x), gu.dev(params)
    loss, grad, ml, mg = (torch.zeros(s, device="cuda") for s in ((B,), (B, P), (1,), (P,)))
    m, v = torch.zeros(P, device="cuda"), torch.zeros(P, device="cuda")
    for step in (1, 2, 3):
        now = pd.cpu().numpy()
        c.qsv_distill_grad(circ, xd, pd, None, gu.dev(idx.astype(np.int32)), gu.dev(logits), loss, grad, ml, mg)
        c.qsv_adam_step(pd, mg, m, v, step, 0.05)
        torch.cuda.synchronize()
        ref = circuit_reference(oracle, spec, n, x, now, None, idx, logits, 1.0, None)
        assert np.all(np.abs(grad.cpu().numpy() - ref[1]).max(axis=1) <= ref[2] + 1e-5)
        assert np.all(np.abs(loss.cpu().numpy() - ref[0]) <= ref[2] + 1e-5)
    c.qsv_amp_encode(xd)
    c.qsv_apply_layers(circ, pd, None, 0)
    u = g.random((B, 12))
    f = dict(top_p=[0.9, 0.6], temperature=[0.7, 1.0], min_p=[0.0, 0.02])
    out, kept = torch.zeros((B, 12), dtype=torch.int64, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    c.qsv_sample(qb.QSV_S_STATE, out, gu.dev(u), kept=kept, **{k: torch.tensor(a, device="cuda") for k, a in f.items()})
    p = torch.zeros((B, 1 << n), device="cuda")
    c.qsv_measure(qb.QSV_M_PROBS, p)
    torch.cuda.synchronize()
    ref = sampled(values_of("probs", p), False, u, f)
    assert np.array_equal(out.cpu().numpy(), ref[0]) and np.array_equal(kept.cpu().numpy(), ref[2])
    c.close()
