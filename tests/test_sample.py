"""qsv_sample against its definition in 64 bits: outcomes, numbers of outcomes left and log-probabilities, at the sizes
and rows where it can go wrong.

Outcomes and numbers have to be equal.  A log-probability is the quotient of two whole numbers that are the same on both
sides but where e_k 2^S lies within 2^-50 of it from the middle between two: then w, or W, which is at least 2^32 here, is
off by 1.  Of an outcome that is drawn w is either that large too, or equal.  So 2^-24 |x| for the rounding to float32 and
2^-31 for the others bound the error.
"""
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
LOGS = ("f32", "f16", "bf16")


# ---- the definition --------------------------------------------------------------------------------------------------
def reference_row(v, logs, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(indices left, ascending; their whole weights) of one row of float64 values."""
    v = np.asarray(v, dtype=np.float64)
    none = np.zeros(0, dtype=np.int64), np.zeros(0, dtype=np.int64)
    if not (0 <= t < INF and top_k >= 0 and 0 <= top_p < INF and 0 <= min_p <= 1):
        return none
    with np.errstate(invalid="ignore"):
        there = np.flatnonzero(v > (-INF if logs else 0.0))
    if not there.size:
        return none
    there = there[np.argsort(-v[there], kind="stable")]      # the lowest index first among equals
    m = v[there[0]]
    scale = 2.0 ** min(51, 62 - (len(v) - 1).bit_length())
    if t == 0:
        return there[:1], np.array([int(scale)])
    with np.errstate(all="ignore"):
        e = np.exp((v[there] - m) / t) if logs else v[there] / m if t == 1 else (v[there] / m) ** (1.0 / t)
    e[v[there] == m] = 1.0
    left, e = there[e >= min_p], e[e >= min_p]
    if top_k:
        left, e = left[:top_k], e[:top_k]
    w = np.rint(e * scale).astype(np.int64)
    if top_p < 1:
        border = -(-int(np.rint(np.float64(np.float32(top_p)) * 2 ** 31)) * int(w.sum()) // 2 ** 31)
        stay = np.cumsum(w) - w < border
        stay[0] = True
        left, w = left[stay], w[stay]
    order = np.argsort(left)
    return left[order], w[order]


def reference(values, logs, uniforms, filters):
    out, logp, kept = [], [], []
    for r, v in enumerate(values):
        f = {k: float(np.float32(x[r])) if k != "top_k" else int(x[r]) for k, x in filters.items()}
        f = {("t" if k == "temperature" else k): x for k, x in f.items()}
        idx, w = reference_row(v, logs, **f)
        kept.append(len(idx))
        run = np.cumsum(w)
        o, lp = [], []
        for u in uniforms[r].tolist():
            if not len(idx) or not 0 <= u < 1:
                o.append(-1)
                lp.append(-INF)
                continue
            t = (math.floor(u * 2 ** 53) * int(run[-1])) >> 53
            at = int(np.searchsorted(run, t, side="right"))
            o.append(int(idx[at]))
            lp.append(math.log(int(w[at]) / int(run[-1])))
        out.append(o)
        logp.append(lp)
    shape = (len(values), uniforms.shape[1])
    return np.array(out, dtype=np.int64).reshape(shape), np.array(logp).reshape(shape), np.array(kept)


# ---- the reference itself, and the refusals, without a device --------------------------------------------------------
def test_reference_small_closed_forms():
    idx, w = reference_row([0.0, math.log(2), 0.0, -INF], True)
    assert idx.tolist() == [0, 1, 2] and w[1] == 2 ** 51 and abs(w[0] - 2 ** 50) <= 1
    assert reference_row([1.0, 3.0, 3.0, 2.0], True, t=0)[0].tolist() == [1]
    assert reference_row([1.0, 3.0, 3.0, 3.0], True, top_k=2)[0].tolist() == [1, 2]
    assert reference_row([1.0, 1.0, 1.0, 1.0], False, top_p=0.5)[0].tolist() == [0, 1]
    assert reference_row([1.0, 1.0, 1.0, 1.0], False, top_p=0.0)[0].tolist() == [0]
    assert reference_row([0.5, 1.0, 0.25, 0.0], False, min_p=0.5)[0].tolist() == [0, 1]
    assert reference_row([NAN, -INF], True)[0].size == 0


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
    L.request_sample.restype = ctypes.c_char_p
    L.request_sample.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64]
    return L


def good(**more):
    r = qb.qsv_sample_req()
    r.kind, r.scores_dev, r.rows, r.cols, r.row_stride = qb.QSV_S_F32, 0x1000, 3, 10, 10
    r.uniforms_dev, r.shots, r.out_dev = 0x2000, 2, 0x3000
    for k, v in more.items():
        setattr(r, k, v)
    return r


def test_refusals(checks):
    say = lambda r, n=4, batch=3: checks.request_sample(ctypes.byref(r) if r is not None else None, n, batch)  # noqa: E731
    assert say(good()) is None
    assert b"NULL" in say(None)
    assert b"reserved" in say(good(reserved=1))
    for kind in (0, 6, -1):
        assert b"kind" in say(good(kind=kind))
    for rows in (-1, (1 << 24) + 1):
        assert b"rows" in say(good(rows=rows))
    for cols in (0, -1, (1 << 30) + 1):
        assert b"cols" in say(good(cols=cols))
    assert b"scores_dev" in say(good(scores_dev=None))
    assert b"aligned" in say(good(scores_dev=0x1002))
    assert say(good(scores_dev=0x1002, kind=qb.QSV_S_F16)) is None
    assert b"aligned" in say(good(scores_dev=0x1001, kind=qb.QSV_S_BF16))
    assert b"row_stride" in say(good(row_stride=9))
    assert b"row_stride" in say(good(row_stride=1 << 37))
    assert say(good(row_stride=0, rows=1)) is None
    assert b"shots" in say(good(shots=-1))
    assert b"shots" in say(good(shots=1 << 31))               # with three rows
    assert b"shots" in say(good(shots=1 << 62))
    assert b"uniforms" in say(good(uniforms_dev=None))
    assert b"out_dev" in say(good(out_dev=None))
    assert say(good(shots=0, uniforms_dev=None, out_dev=None)) is None
    assert say(good(rows=0, scores_dev=None, uniforms_dev=None, out_dev=None)) is None
    state = dict(kind=qb.QSV_S_STATE, scores_dev=None, rows=3, cols=16)
    assert say(good(**state)) is None
    assert b"state" in say(good(**dict(state, scores_dev=0x1000)))
    assert b"state" in say(good(**dict(state, cols=8)))
    assert b"state" in say(good(**dict(state, rows=2)))
    assert qb.load().qsv_sample(None, ctypes.byref(good())) == qb.QSV_ERR_INVALID_ARG


def test_workspace_sizes():
    assert qb.qsv_sample_workspace_bytes(-1, 5) == 0 == qb.qsv_sample_workspace_bytes(5, 0)
    assert 0 < qb.qsv_sample_workspace_bytes(0, 5) <= qb.qsv_sample_workspace_bytes(1, 1 << 20) < qb.qsv_sample_workspace_bytes(1, 1 << 30)
    assert ctypes.sizeof(qb.qsv_sample_req) == 112


# ---- on the GPU ------------------------------------------------------------------------------------------------------
def kinds():
    return {"f32": qb.QSV_S_F32, "f16": qb.QSV_S_F16, "bf16": qb.QSV_S_BF16, "probs": qb.QSV_S_PROBS}


def torch_type(src):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "probs": torch.float32}[src]


@pytest.fixture(scope="module")
def ctx():
    c = qb.Context(1, 1)
    yield c
    c.close()


def on_gpu(ctx, src, scores, uniforms, filters, logp=True, kept=True):
    import torch
    rows, shots = uniforms.shape
    f = {k: torch.as_tensor(x, dtype=torch.int32 if k == "top_k" else torch.float32).cuda() for k, x in filters.items()}
    out = torch.full((rows, shots), -7, dtype=torch.int64, device="cuda")
    lp = torch.full((rows, shots), 7.0, device="cuda") if logp else None
    kp = torch.full((rows,), -7, dtype=torch.int32, device="cuda") if kept else None
    ctx.qsv_sample(kinds()[src] if src != "state" else qb.QSV_S_STATE, out, torch.as_tensor(uniforms).cuda(),
                   scores=None if src == "state" else scores, logp=lp, kept=kp, **f)
    torch.cuda.synchronize()
    return out.cpu().numpy(), lp.cpu().numpy() if logp else None, kp.cpu().numpy() if kept else None


def same(got, ref):
    out, logp, kept = got
    assert np.array_equal(out, ref[0])
    if kept is not None:
        assert np.array_equal(kept, ref[2])
    if logp is not None:
        with np.errstate(invalid="ignore"):
            close = np.abs(logp - ref[1]) <= 2.0 ** -24 * np.abs(ref[1]) + 2.0 ** -31
        assert np.all(close | (logp == ref[1]))


def values_of(src, scores):
    """The float64 values that the kernel sees."""
    return scores.float().cpu().numpy().astype(np.float64) + 0.0


EACH = dict(temperature=[0.0, 0.6, 1.0, 1.0, 1.7, 1.0, 0.8], top_k=[0, 3, 0, 1, 40, 0, 5], top_p=[1.0, 0.9, 0.8, 1.0, 0.95, 0.3, 0.0],
            min_p=[0.0, 0.0, 0.05, 0.0, 0.01, 0.0, 0.2])


def spread(filters, rows):
    return {k: [v[r % len(v)] for r in range(rows)] for k, v in filters.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16", "probs"])
@pytest.mark.parametrize("cols", [1, 2, 3, 63, 64, 65, 255, 257, 511, 512, 513, 1000, 2049, 4099, 8191, 8192, 8193, 20001])
def test_sizes(ctx, src, cols):
    import torch
    g = torch.Generator().manual_seed(cols)
    rows, shots = 7, 9
    z = torch.randn((rows, cols + 3), generator=g) * 3
    if src == "probs":
        z = z.exp()
    scores = z.to(torch_type(src)).cuda()[:, :cols]
    u = torch.rand((rows, shots), generator=g, dtype=torch.float64).numpy()
    for filters in ({}, spread(EACH, rows), dict(top_k=[2] * rows), dict(top_p=[0.7] * rows), dict(min_p=[0.1] * rows)):
        same(on_gpu(ctx, src, scores, u, filters), reference(values_of(src, scores), src in LOGS, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16", "probs"])
@pytest.mark.parametrize("cols", [37, 700, 9000])
def test_values_at_the_edges(ctx, src, cols):
    """Masked outcomes of every kind, rows of nothing but them, ties, infinities, zeros of both signs, the type's range."""
    import torch
    g = torch.Generator().manual_seed(7)
    t, u = torch_type(src), torch.rand((12, 5), generator=g, dtype=torch.float64).numpy()
    u[:, 0] = 0.0
    u[:, 1] = 1.0 - 2.0 ** -53
    z = torch.randn((12, cols), generator=g) * 2
    low, high = torch.finfo(t).min, torch.finfo(t).max
    z[0] = -INF
    z[1] = NAN
    z[2] = low                                          # an ordinary score, as long as nothing else is there
    z[3, 1:] = -INF
    z[4] = 0.0
    z[4, ::2] = -0.0
    z[5] = torch.round(z[5])                            # many ties
    z[6, cols // 2] = INF
    z[6, 3] = INF
    z[7, ::2] = low
    z[7, 1::4] = NAN
    z[8] = high
    z[8, 5] = low
    z[9] = torch.finfo(t).tiny * torch.randint(1, 5, (cols,), generator=g)
    z[10, :-1] = -INF
    z[11] = 1.0
    scores = z.to(t).cuda()
    for filters in ({}, dict(temperature=[0.0] * 12), dict(top_k=[4] * 12), dict(top_p=[0.5] * 12), dict(min_p=[1.0] * 12),
                    dict(temperature=[0.5] * 12, top_k=[6] * 12, top_p=[0.75] * 12, min_p=[0.001] * 12),
                    dict(temperature=[1e-30] * 12, top_p=[0.9] * 12), dict(temperature=[3e38] * 12, top_k=[9] * 12)):
        same(on_gpu(ctx, src, scores, u, filters), reference(values_of(src, scores), src in LOGS, u, filters))


@pytest.mark.gpu
def test_parameters_out_of_range_and_uniforms_outside(ctx):
    import torch
    z = torch.randn((10, 300), generator=torch.Generator().manual_seed(3)).cuda()
    u = np.tile(np.array([0.25, -0.1, 1.0, NAN, 0.75]), (10, 1))
    filters = dict(temperature=[1.0, -1.0, NAN, INF, 1, 1, 1, 1, 1, 1], top_k=[0, 0, 0, 0, -1, 0, 0, 0, 0, 2**31 - 1],
                   top_p=[1, 1, 1, 1, 1, -0.5, NAN, 1, 1, 5.0], min_p=[0, 0, 0, 0, 0, 0, 0, 1.5, NAN, 0])
    got = on_gpu(ctx, "f32", z, u, filters)
    same(got, reference(values_of("f32", z), True, u, filters))
    assert got[2].tolist() == [300] + [0] * 8 + [300]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 300001), (2, 262147), (3, 524288)])
@pytest.mark.parametrize("src", ["f32", "bf16", "probs"])
def test_long_rows(ctx, src, rows, cols):
    import torch
    g = torch.Generator().manual_seed(cols)
    z = torch.randn((rows, cols), generator=g) * 2
    z = (z.exp() if src == "probs" else z).to(torch_type(src)).cuda()
    for shots in (3, 40):
        u = torch.rand((rows, shots), generator=g, dtype=torch.float64).numpy()
        for filters in ({}, dict(top_k=[1000] * rows), dict(top_p=[0.9] * rows), spread(EACH, rows),
                        dict(top_k=[100000] * rows, top_p=[0.99] * rows, min_p=[1e-4] * rows)):
            same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), src in LOGS, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [5000, 270000])
def test_rows_of_near_equal_values(ctx, cols):
    """Cuts that fall between neighbouring values, and among equals, of which every bin is full."""
    import torch
    g = torch.Generator().manual_seed(1)
    base = np.float32(1.0) + np.arange(5, dtype=np.float32) * np.float32(2.0 ** -23)
    z = torch.from_numpy(base)[torch.randint(5, (3, cols), generator=g)].cuda()
    z[1] = 1.0
    z[2] *= 1e-38
    u = torch.rand((3, 6), generator=g, dtype=torch.float64).numpy()
    for src in ("f32", "probs"):
        for filters in (dict(top_k=[cols // 3] * 3), dict(top_p=[0.61] * 3), dict(top_k=[cols // 2] * 3, top_p=[0.5] * 3)):
            same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), src in LOGS, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
def test_the_longest_rows(src):
    """Two rows of 2^30, more than 2^32 bytes to the second one's start; few scores are not masked."""
    import torch
    cols, stride = 1 << 30, (1 << 30) + 5
    c = qb.Context(1, 1, ws_bytes=max(qb.qsv_workspace_bytes(1, 1), qb.qsv_sample_workspace_bytes(2, cols)))
    flat = torch.full((2 * stride,), -np.inf, dtype=torch_type(src), device="cuda")
    scores = flat[:2 * stride].view(2, stride)[:, :cols]
    at = np.array([0, 3, cols // 3, cols - 2, cols - 1])
    v = np.array([[0.5, -1.0, 2.0, 1.5, -0.25], [1.0, 1.0, -3.0, 0.75, 1.0]])
    for r in range(2):
        for k, x in zip(at, v[r]):
            scores[r, int(k)] = float(x)
    u = np.random.default_rng(3).random((2, 40))
    for filters in ({}, dict(top_k=[3, 2]), dict(top_p=[0.9, 0.6]), dict(temperature=[0.0, 0.7])):
        # the few among few (whose weights have more bits; no border is that near)
        few = np.full((2, 6), -np.inf)
        few[:, :5] = v
        ref = reference(few, True, u, filters)
        out = np.where(ref[0] >= 0, at[np.minimum(ref[0], 4)], -1)
        same(on_gpu(c, src, scores, u, filters), (out, ref[1], ref[2]))
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [9000, 270000])
@pytest.mark.parametrize("src,high,low", [("f32", 0x3b1fffff, 0xfffff), ("bf16", 0x3b1f, 0xf), ("f16", 0x18ff, 0x7)])
def test_cuts_right_below_zero(ctx, src, high, low, cols):
    """Scores about 0 in one bin, whose keys are parted right between those of -0 and 0: the highest key is chosen for that.  The
    cut falls among the negative ones, with many zeros (of both signs) beside it."""
    import torch
    g = np.random.default_rng(cols)
    sign = 1 << (31 if src == "f32" else 15)
    what = g.integers(0, 10, (4, cols))
    bits = np.where(what < 2, g.integers(high // 2, high, (4, cols)), np.where(what < 6, 0, sign | g.integers(1, low + 1, (4, cols))))
    bits = np.where(what == 5, sign, bits)
    bits[:, 7] = high
    word = bits.astype(np.uint32).view(np.int32) if src == "f32" else bits.astype(np.uint16).view(np.int16)
    z = torch.from_numpy(word).view(torch_type(src)).cuda()
    u = g.random((4, 6))
    k = [cols * 7 // 10, cols * 6 // 10 + 3, cols * 8 // 10, cols * 9 // 10]
    for filters in (dict(top_k=k), dict(top_p=[0.7, 0.65, 0.8, 0.95]), dict(top_k=k, top_p=[0.99, 0.95, 0.9, 0.8])):
        same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), True, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [300, 1000, 8192, 9000, 60000, 270000])
@pytest.mark.parametrize("src,m,t", [("bf16", 200.0, 0.11), ("bf16", 40.0, 0.028), ("bf16", -200.0, 0.1), ("bf16", 3e38, 1.3e35),
                                     ("f16", 2000.0, 0.11), ("f16", 60000.0, 1.6), ("f16", -40.0, 0.002), ("f16", 4e-7, 4e-9)])
def test_scores_whose_spacing_is_many_temperatures(ctx, src, m, t, cols):
    """Two neighbouring scores of 16 bits lie so far apart that the next below the lowest with a weight is more than 63 factors of two
    from the highest.  One of the highest, many one and two spacings below, and top-p without top-k: cuts in every one of them."""
    import torch
    g = np.random.default_rng(cols)
    word = int(torch.tensor([m], dtype=torch_type(src)).view(torch.int16).item()) & 0xffff
    down = lambda d: word - d if m > 0 else word + d  # noqa: E731
    bits = np.full((6, cols), down(40) if m < 0 or word > 40 else 0)
    bits[:, 7] = word
    for d, many in ((1, 20), (2, 200), (3, 30), (5, 30)):
        for r in range(6):
            bits[r, 10 + g.permutation(cols - 10)[:min(many, cols // 8)]] = down(min(d, word - 1))
    bits[1, 11] = bits[2, cols - 1] = word
    z = torch.from_numpy(bits.astype(np.uint16).view(np.int16)).view(torch_type(src)).cuda()
    for shots in (1, 40):
        u = g.random((6, shots))
        for top_p in ([0.999] * 6, [1 - 2.0 ** -20] * 6, [0.5, 0.9, 0.99, 0.9999, 0.99999, 0.0]):
            for more in ({}, dict(min_p=[0.0, 1e-9, 1e-4, 0.0, 1e-30, 0.5])):
                filters = dict(temperature=[t] * 6, top_p=top_p, **more)
                same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), True, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [40, 300, 9000, 270000])
def test_probabilities_over_the_whole_range_at_high_temperatures(ctx, cols):
    """Values from the smallest number that float32 holds to the largest, 2^277 apart: at T = 8 the lowest still weigh 2^-35."""
    import torch
    g = np.random.default_rng(cols)
    v = np.exp2(g.uniform(-149, 127.9, (6, cols))).astype(np.float32)
    v[:, 0], v[:, 1], v[:, 2] = 2.0 ** -149, 3e38, 2.0 ** -120
    v[1, 3:] = 2.0 ** -149                        # all but three at the lowest
    v[2, 3:] = 2.0 ** -110
    z = torch.from_numpy(v).cuda()
    t = [8.0, 8.0, 4.0, 5.5, 16.0, 1000.0]
    for shots in (3, 40):
        u = g.random((6, shots))
        for filters in (dict(temperature=t), dict(temperature=t, top_p=[0.999, 0.9, 0.9999, 0.8, 0.5, 0.97]),
                        dict(temperature=t, top_k=[cols - 1, 5, cols // 2, 0, 7, 30], top_p=[0.9999] * 6),
                        dict(temperature=t, min_p=[1e-11, 1e-10, 1e-18, 0.01, 1e-6, 0.9])):
            same(on_gpu(ctx, "probs", z, u, filters), reference(values_of("probs", z), False, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f16", "f32"])
def test_a_row_does_not_depend_on_its_alignment(ctx, src):
    import torch
    g = torch.Generator().manual_seed(5)
    flat = (torch.randn(70000, generator=g) * 3).to(torch_type(src)).cuda()
    u = torch.rand((2, 4), generator=g, dtype=torch.float64).numpy()
    filters = dict(top_k=[50, 0], top_p=[0.9, 0.95])
    for cols in (5, 600, 30000):
        for off in range(5):
            z = torch.as_strided(flat, (2, cols), (cols + 7, 1), off)
            same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), True, u, filters))


@pytest.mark.gpu
@pytest.mark.parametrize("n,batch", [(1, 3), (4, 5), (9, 4), (14, 2), (19, 1)])
def test_state(n, batch):
    import torch
    g = torch.Generator().manual_seed(n)
    c = qb.Context(n, batch)
    a = torch.randn((batch, 1 << n, 2), generator=g)
    a[0, ::3] = 0.0
    c.state.copy_(a / a.square().sum(dim=(1, 2), keepdim=True).sqrt())
    p = torch.zeros((batch, 1 << n), device="cuda")
    c.qsv_measure(qb.QSV_M_PROBS, p)
    u = torch.rand((batch, 21), generator=g, dtype=torch.float64).numpy()
    before = c.state.clone()
    for filters in ({}, dict(temperature=[0.5] * batch), spread(EACH, batch), dict(top_p=[0.8] * batch)):
        ref = reference(values_of("probs", p), False, u, filters)
        same(on_gpu(c, "state", None, u, filters), ref)
        same(on_gpu(c, "probs", p, u, filters), ref)
    assert torch.equal(c.state, before)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16", "probs"])
@pytest.mark.parametrize("rows,cols,shots", [(3, 9000, 33), (2, 70001, 200), (300, 8193, 40), (300, 9999, 3)])
def test_many_shots_and_many_rows(ctx, src, rows, cols, shots):
    """Rows whose shots another launch draws, and more rows than there are CUs; all kinds of cuts side by side."""
    import torch
    g = torch.Generator().manual_seed(rows + cols)
    z = torch.randn((rows, cols), generator=g) * 2
    z[rows // 2] = -INF if src in LOGS else 0.0
    z = (z.exp() if src == "probs" else z).to(torch_type(src)).cuda()
    u = torch.rand((rows, shots), generator=g, dtype=torch.float64).numpy()
    u[0, 1] = 1.5
    for filters in ({}, spread(EACH, rows), dict(top_p=[0.97] * rows, temperature=[1.5] * rows)):
        same(on_gpu(ctx, src, z, u, filters), reference(values_of(src, z), src in LOGS, u, filters))


@pytest.mark.gpu
def test_outputs_left_out_and_shots_of_none(ctx):
    import torch
    z = torch.randn((3, 400), generator=torch.Generator().manual_seed(2)).cuda()
    u = np.full((3, 2), 0.4)
    ref = reference(values_of("f32", z), True, u, dict(top_k=[5] * 3))
    got = on_gpu(ctx, "f32", z, u, dict(top_k=[5] * 3), logp=False, kept=False)
    assert np.array_equal(got[0], ref[0])
    kept = torch.zeros(3, dtype=torch.int32, device="cuda")
    none = torch.zeros((3, 0), dtype=torch.int64, device="cuda")
    ctx.qsv_sample(qb.QSV_S_F32, none, torch.zeros((3, 0), dtype=torch.float64, device="cuda"), scores=z,
                   top_k=torch.full((3,), 5, dtype=torch.int32, device="cuda"), kept=kept)
    ctx.qsv_sample(qb.QSV_S_F32, none[:0], torch.zeros((0, 0), dtype=torch.float64, device="cuda"), scores=z[:0])
    torch.cuda.synchronize()
    assert kept.tolist() == [5, 5, 5]


@pytest.mark.gpu
def test_workspace_refused_before_anything_runs():
    import torch
    c = qb.Context(1, 1)
    rows, cols = 2000, 300000              # more rows of histograms than this context's workspace holds
    assert qb.qsv_sample_workspace_bytes(rows, cols) > c.ws.numel()
    out = torch.full((rows, 1), -7, dtype=torch.int64, device="cuda")
    z = torch.zeros((1, cols), device="cuda").expand(rows, cols)
    r = qb.qsv_sample_req()
    u = torch.zeros((rows, 1), dtype=torch.float64, device="cuda")
    r.kind, r.scores_dev, r.rows, r.cols, r.row_stride = qb.QSV_S_F32, z.data_ptr(), rows, cols, cols
    r.uniforms_dev, r.shots, r.out_dev = u.data_ptr(), 1, out.data_ptr()
    assert c.L.qsv_sample(c.h, ctypes.byref(r)) == qb.QSV_ERR_WORKSPACE
    torch.cuda.synchronize()
    assert int((out != -7).sum()) == 0
    c.close()


@pytest.mark.gpu
def test_few_shots_need_no_workspace():
    """More rows than the context's workspace has room for the weights of, which only many shots need."""
    import torch
    c = qb.Context(1, 1)
    rows, cols = 140000, 8200
    assert qb.qsv_sample_workspace_bytes(rows, cols) > qb.qsv_workspace_bytes(1, 1)
    z = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    at = torch.randint(0, cols, (rows, 1), generator=torch.Generator().manual_seed(4)).cuda()
    z.scatter_(1, at, torch.tensor(40.0, dtype=torch.bfloat16, device="cuda").expand(rows, 1))
    f = dict(top_p=torch.full((rows,), 0.5, device="cuda"))
    kept = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for shots, fits in ((1, True), (32, True), (33, False)):
        out = torch.full((rows, shots), -7, dtype=torch.int64, device="cuda")
        u = torch.rand((rows, shots), dtype=torch.float64, device="cuda")
        if fits:
            c.qsv_sample(qb.QSV_S_BF16, out, u, scores=z, kept=kept, **f)
            assert bool((out == at).all()) and bool((kept == 1).all())
        else:
            with pytest.raises(qb.QsvError) as refused:
                c.qsv_sample(qb.QSV_S_BF16, out, u, scores=z, **f)
            assert refused.value.status == qb.QSV_ERR_WORKSPACE and bool((out == -7).all())
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [3000, 20000, 300000])
def test_replays_of_a_captured_call(cols):
    """New scores and uniforms between the replays; eager calls of the same context in between."""
    import torch
    g = torch.Generator().manual_seed(11)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = qb.Context(1, 1)
        z = torch.zeros((2, cols), device="cuda")
        u = torch.zeros((2, 50), dtype=torch.float64, device="cuda")
        out = torch.zeros((2, 50), dtype=torch.int64, device="cuda")
        kept = torch.zeros(2, dtype=torch.int32, device="cuda")
        f = dict(top_p=torch.full((2,), 0.9, device="cuda"), top_k=torch.full((2,), 500, dtype=torch.int32, device="cuda"))
        call = lambda: c.qsv_sample(qb.QSV_S_F32, out, u, scores=z, kept=kept, **f)  # noqa: E731
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for i in range(4):
            z.copy_(torch.randn((2, cols), generator=g) * (i + 1))
            u.copy_(torch.rand((2, 50), generator=g, dtype=torch.float64))
            out.fill_(-7)
            graph.replay()
            stream.synchronize()
            got = out.cpu().numpy(), None, kept.cpu().numpy()
            same(got, reference(values_of("f32", z), True, u.cpu().numpy(), dict(top_p=[0.9] * 2, top_k=[500] * 2)))
            out.fill_(-7)
            call()
            stream.synchronize()
            assert np.array_equal(out.cpu().numpy(), got[0])
        c.close()
