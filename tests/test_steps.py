"""qsv_clip_grads and qsv_adam_clipped against their formulas in 64 bits.

Errors that the kernels may make: squares and sums in float64, so N is off by 2^-53 times the number of values (2^-27 at 2^26 of
them) before it is rounded to float32 (2^-24); f and the products in float64; every value is rounded to float32 and to its type:
half a step of each.  Adam's values are rounded once to float32 from float64, m and v from terms of one sign or of their own size."""
import ctypes
import math
import os
import shutil
import subprocess
import time

import numpy as np
import pytest

from paper_2602_13140_amd import binding as qb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF, NAN = math.inf, math.nan
U = 2.0 ** -24


def tt(src):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[src]


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
    L.request_clip.restype = L.request_adam.restype = ctypes.c_char_p
    L.request_clip.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_double]
    L.request_adam.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_double]
    return L


def tensors(*rows):
    """(address, rows, cols, stride[, kind]) each."""
    a = (qb.qsv_tensor * max(1, len(rows)))()
    for e, r in zip(a, rows):
        e.data_dev, e.rows, e.cols, e.row_stride = r[:4]
        e.kind = r[4] if len(r) > 4 else qb.QSV_S_F32
    return a


def test_refusals_of_clipping(checks):
    def say(grads, outs=None, norm=1.0, n=None):
        return checks.request_clip(grads, outs, len(grads) if n is None else n, norm)
    one = (0x1000, 1, 100, 0)
    assert say(tensors(one)) is None and say(tensors(one), norm=INF) is None and say(tensors(one), norm=0.0) is None
    assert say(None, n=0) is None and b"NULL" in say(None, n=2) and b"4096" in say(tensors(one), n=-1) and b"4096" in say(tensors(one), n=4097)
    for m in (-1.0, NAN):
        assert b"max_norm" in say(tensors(one), norm=m)
    for bad, why in (((0x1000, -1, 5, 5), b"rows"), ((0x1000, 5, -1, 5), b"rows"), ((0x1000, 1 << 30, 1 << 30, 1 << 30), b"2^38"), ((None, 1, 5, 0), b"NULL"),
                     ((0x1002, 1, 5, 0), b"aligned"), ((0x1000, 2, 5, 4), b"row_stride"), ((0x1000, 1, 5, 0, 4), b"kind"), ((0x1001, 1, 5, 0, qb.QSV_S_F16), b"aligned")):
        assert why in say(tensors(bad)) and why in say(tensors(one), tensors(bad)) or b"shapes" in say(tensors(one), tensors(bad))
    t = tensors(one)
    t[0].reserved = 1
    assert b"reserved" in say(t)
    assert say(tensors((None, 0, 5, 0), (None, 5, 0, 0))) is None
    half = 1 << 37
    assert say(tensors((0x1000, 1, half, 0), (0x1000 + 4 * half, 1, half, 0))) is None
    assert b"2^38" in say(tensors((0x1000, 1, half, 0), (0x1000 + 4 * half, 1, half, 0), (0x1000 + 8 * half, 1, 1, 0)))
    twice = tensors(one, one)
    assert b"overlap" in say(twice) and say(twice, norm=INF) is None                     # scaled twice, or read only
    assert b"overlap" in say(tensors(one, (0x1000 + 396, 1, 8, 0))) and say(tensors(one, (0x1000 + 400, 1, 8, 0))) is None
    cols = tensors((0x1000, 10, 6, 16), (0x1000 + 24, 10, 10, 16))                       # columns of one buffer
    assert say(cols) is None and b"overlap" in say(tensors((0x1000, 10, 7, 16), (0x1000 + 24, 10, 10, 16)))
    assert say(tensors((0x1000 + 24, 10, 10, 16), (0x1000 + 64, 9, 6, 16))) is None
    assert b"overlap" in say(tensors((0x1000, 10, 6, 16), (0x1000 + 24, 10, 10, 17)))
    far = tensors((0x9000, 1, 100, 0))
    assert say(tensors(one), far) is None and say(tensors(one), tensors(one)) is None
    for other in ((0x9000, 2, 50, 50), (0x9000, 1, 99, 0), (0x9000, 1, 100, 0, qb.QSV_S_BF16)):
        assert b"shapes" in say(tensors(one), tensors(other))
    assert b"overlap" in say(tensors(one), tensors((0x1004, 1, 100, 0)))
    two = tensors(one, (0x5000, 1, 100, 0))
    assert b"overlap" in say(two, tensors((0x5000, 1, 100, 0), (0x9000, 1, 100, 0)))     # another's gradient
    assert b"overlap" in say(two, tensors((0x9000, 1, 100, 0), (0x9000, 1, 100, 0)))
    assert b"overlap" in say(tensors((0x1000, 4, 10, 12)), tensors((0x1000, 4, 10, 13)))
    assert qb.load().qsv_clip_grads(None, two, None, 2, 1.0, None) == qb.QSV_ERR_INVALID_ARG


def test_refusals_of_destinations(checks):
    """Of outs that have their gradients' kind and shape: what is wrong with an address, a stride or a field is said, also behind a good one and
    where nothing would be scaled."""
    def say(grad, out, norm=1.0, reserved=0):
        good = (0x40000, 1, 100, 0), (0x50000, 1, 100, 0)
        outs = tensors(good[1], out)
        outs[1].reserved = reserved
        return checks.request_clip(tensors(good[0], grad), outs, 2, norm)
    for norm in (0.0, 1.0, INF):
        for kind, size in ((qb.QSV_S_F32, 4), (qb.QSV_S_F16, 2), (qb.QSV_S_BF16, 2)):
            vector, rows = (0x1000, 1, 100, 0, kind), (0x1000, 4, 10, 12, kind)
            assert say(vector, (0x9000, 1, 100, 0, kind), norm) is None and say(rows, (0x9000, 4, 10, 10, kind), norm) is None
            for grad in (vector, rows):
                shape = grad[1:4] + (kind,)
                assert b"data_dev is NULL" in say(grad, (None,) + shape, norm)
                for off in range(1, size):
                    assert b"data_dev must be aligned" in say(grad, (0x9000 + off,) + shape, norm)
                assert b"reserved must be 0" in say(grad, (0x9000,) + shape, norm, reserved=1)
            for stride in (-1, 0, 9, (1 << 38) + 1):
                assert b"row_stride must be in" in say(rows, (0x9000, 4, 10, stride, kind), norm)
            for shape in ((1, 99, 0), (2, 50, 50), (100, 1, 1), (1, 101, 0)):
                assert b"shapes" in say(vector, (0x9000,) + shape + (kind,), norm)
            assert b"shapes" in say(vector, (0x9000, 1, 100, 0, qb.QSV_S_F16 if size == 4 else qb.QSV_S_F32), norm)
            assert b"kind must be one" in say(vector, (0x9000, 1, 100, 0, 4), norm)
            assert b"rows and cols" in say(vector, (0x9000, -1, 100, 0, kind), norm)


def test_refusals_of_adam(checks):
    def lists(*rows):
        a = (qb.qsv_adam_tensor * max(1, len(rows)))()
        for e, r in zip(a, rows):
            e.param_dev, e.grad_dev, e.m_dev, e.v_dev, e.count = r[:5]
            e.kind = r[5] if len(r) > 5 else qb.QSV_S_F32
        return a
    say = lambda a, n=None, m=1.0: checks.request_adam(a, len(a) if n is None else n, m)  # noqa: E731
    one = (0x1000, 0x2000, 0x3000, 0x4000, 100)
    assert say(lists(one)) is None and say(None, 0) is None and b"NULL" in say(None, 1) and b"4096" in say(lists(one), 4097)
    assert b"max_norm" in say(lists(one), m=-0.5) and say(lists(one), m=INF) is None
    far = [1 << 44, 2 << 44, 3 << 44, 4 << 44]
    assert say(lists((*far, 1 << 38))) is None and b"2^38" in say(lists((*far, 1 << 38), (*[5 * x for x in far], 1)))
    assert say(lists((None, None, None, None, 0))) is None and b"count" in say(lists(one[:4] + (-1,)))
    for i in range(4):
        assert b"NULL" in say(lists(one[:i] + (None,) + one[i + 1:])) and b"aligned" in say(lists(one[:i] + (one[i] + 2,) + one[i + 1:]))
        for j in range(i):
            assert b"overlap" in say(lists(one[:i] + (one[j],) + one[i + 1:])) and b"overlap" in say(lists(one[:i] + (one[j] + 396,) + one[i + 1:]))
    assert say(lists(one[:1] + (0x2002,) + one[2:] + (qb.QSV_S_BF16,))) is None and b"kind" in say(lists(one + (5,)))
    shared = (0x5000, 0x2000, 0x6000, 0x7000, 100)                                       # one gradient for two tensors: read only
    assert say(lists(one, shared)) is None and b"overlap" in say(lists(one, (0x5000, 0x8000, 0x3000, 0x7000, 100)))
    assert qb.load().qsv_adam_clipped(None, lists(one), 1, 1, 0.1, 0.9, 0.999, 1e-8, 1.0, None) == qb.QSV_ERR_INVALID_ARG


def test_overlaps_against_every_byte(checks):
    """Spans at random: what is let through has no byte twice, and of single rows nothing else is refused."""
    g = np.random.default_rng(1)
    let = 0
    for _ in range(3000):
        n = int(g.integers(2, 5))
        stride = int(g.integers(4, 9))
        rows = []
        for _ in range(n):
            cols = int(g.integers(1, 4))
            rows.append((0x1000 + 4 * int(g.integers(0, 24)), int(g.choice([1, 1, 2, 3])), cols, stride if g.random() < 0.8 else max(cols, int(g.integers(1, 9)))))
        said = checks.request_clip(tensors(*rows), None, n, 1.0)
        words = [a // 4 + r * s + c for a, k, m, s in rows for r in range(k) for c in range(m)]
        if said is None:
            let += 1
            assert len(words) == len(set(words)), rows
        elif all(r[1] == 1 for r in rows):
            assert len(words) != len(set(words)), rows
    assert let > 300


def test_rows_between_other_rows(checks):
    """A single row beside columns of its buffer (whatever its stride says), rows at a multiple of the others' stride: what is refused is what
    overlaps, of lists whose rows have one stride."""
    say = lambda *t: checks.request_clip(tensors(*t), None, len(t), 1.0)  # noqa: E731
    columns = (0x1000, 5, 6, 16)
    assert say(columns, (0x1000 + 24, 1, 10, 0)) is None and say(columns, (0x1000 + 24 + 64, 1, 10, 999)) is None
    assert b"overlap" in say(columns, (0x1000 + 24, 1, 11, 0)) and b"overlap" in say(columns, (0x1000 + 20, 1, 10, 0))
    assert say((0x1000 + 24, 1, 10, 0), columns, (0x1000 + 24 + 64, 1, 4, 3), (0x1000 + 24 + 64 + 16, 1, 6, 0)) is None
    assert say(columns, (0x1000 + 24, 3, 10, 32)) is None and b"overlap" in say(columns, (0x1000 + 24, 3, 11, 32))      # every other row of the rest
    assert say((0x1000, 3, 16, 32), (0x1000 + 64, 1, 16, 16)) is None and say((0x1000, 3, 16, 32), (0x1000 + 64, 2, 16, 32)) is None
    g = np.random.default_rng(5)
    let = refused = 0
    for trial in range(6000):
        n, stride, wide = int(g.integers(2, 6)), int(g.integers(3, 12)), int(g.choice([20, 60, 150]))
        rows = []
        for _ in range(n):
            k, m = int(g.choice([1, 1, 2, 3, 5])), int(g.integers(1, 4))
            rows.append((0x1000 + 4 * int(g.integers(0, wide)), k, m, stride if k > 1 else int(g.integers(0, 20))))
        words = [a // 4 + r * s + c for a, k, m, s in rows for r in range(k) for c in range(m)]
        fine = len(words) == len(set(words))
        assert (say(*rows) is None) == fine, (trial, rows)
        let, refused = let + fine, refused + (not fine)
    assert let > 1000 and refused > 1000


def test_rows_that_would_wrap_around(checks):
    """Extents that 64 bits do not hold would pass as small ones, and what they cover as free."""
    say = lambda *t: checks.request_clip(tensors(*t), None, len(t), 1.0)  # noqa: E731
    for rows, stride in (((1 << 26) + 1, 1 << 38), ((1 << 38), 1 << 38), ((1 << 36) + 1, 1 << 26), ((1 << 18) + 2, 1 << 38)):
        assert b"2^56" in say((0x1000, rows, 1, stride)), (rows, stride)
        assert b"2^56" in say((0x1000, rows, 1, stride), (0x1000 + 4 * stride, 1, 1, 0))
    assert say((0x1000, (1 << 18) + 1, 1, 1 << 38)) is None and say((0x1000, 1 << 38, 1, 1)) is None
    assert b"overlap" in say((0x1000, (1 << 18) + 1, 1, 1 << 38), (0x1000 + (1 << 58), 1, 1, 0))


def test_many_columns_of_one_buffer(checks):
    """A list as long as it may be: what is apart is let through, one word too many is refused, and the time grows with the list, not with its
    square (64 times from 512 tensors to 4096, against 11 of a sort)."""
    def columns(n, wide=4, over=-1, base=0x1000):
        return tensors(*[(base + 4 * wide * i, 8, wide + (i == over), wide * n) for i in range(n)])

    def best(grads, outs):
        took = INF
        for _ in range(5):
            start = time.perf_counter()
            assert checks.request_clip(grads, outs, len(grads), 1.0) is None
            took = min(took, time.perf_counter() - start)
        return took
    for outs in (None, 0x1000, 0x10000000):
        few, many = (best(columns(n), outs and columns(n, base=outs)) for n in (512, 4096))
        assert many < 24 * few, (few, many)
    for over in (0, 17, 4094):
        assert b"overlap" in checks.request_clip(columns(4096, over=over), None, 4096, 1.0)
    assert checks.request_clip(columns(4096, over=4095), None, 4096, 1.0) is not None       # into the next row of the first
    # blocks of a buffer, and a row that reaches from one into the next
    blocks = [(0x1000 + 4 * (64 * 8 * 6 * j + 6 * i), 8, 6, 64 * 6) for j in range(8) for i in range(64)]
    assert checks.request_clip(tensors(*blocks), None, 512, 1.0) is None
    for i in (0, 100, 447):
        assert b"overlap" in checks.request_clip(tensors(*[(b[0], b[1] + (k == i)) + b[2:] for k, b in enumerate(blocks)]), None, 512, 1.0)


def test_overlaps_of_outs_against_every_byte(checks):
    """Gradients and where they go, at random: nothing is let through where a written word comes twice but for a tensor's own; of single
    rows nothing else is refused."""
    g = np.random.default_rng(3)
    let = own = 0
    for trial in range(6000):
        n, wide, stride = int(g.integers(1, 5)), int(g.choice([24, 60, 400])), int(g.integers(4, 9))
        rows, outs = [], []
        for _ in range(n):
            k, m, s = int(g.choice([1, 1, 2, 3])), int(g.integers(1, 4)), stride if g.random() < 0.8 else int(g.integers(4, 9))
            rows.append((0x1000 + 4 * int(g.integers(0, wide)), k, m, s))
            outs.append(rows[-1] if g.random() < 0.3 else (0x1000 + 4 * int(g.integers(0, wide)), k, m, stride))
        said = checks.request_clip(tensors(*rows), tensors(*outs), n, float(g.choice([1.0, INF])))
        words = lambda t: [t[0] // 4 + r * t[3] + c for r in range(t[1]) for c in range(t[2])]  # noqa: E731
        to = [w for t in outs for w in words(t)]
        same = lambda a, b: a[:3] == b[:3] and (a[1] == 1 or a[3] == b[3])                      # noqa: E731
        fine = len(to) == len(set(to)) and all(not set(words(a)) & set(words(b)) or (i == j and same(a, b))
                                               for i, a in enumerate(rows) for j, b in enumerate(outs))
        if said is None:
            assert fine, trial
            let += 1
            own += any(same(a, b) for a, b in zip(rows, outs))
        elif all(t[1] == 1 for t in rows):
            assert not fine, trial
    assert let > 500 and own > 100


def test_overlaps_of_adam_against_every_byte(checks):
    """Parameters, moments and gradients at random, in any order: nothing is let through where a written byte comes twice, nothing else refused."""
    g = np.random.default_rng(2)
    let = 0
    for trial in range(4000):
        n = int(g.integers(1, 5))
        a = (qb.qsv_adam_tensor * n)()
        written, read = [], []
        wide = int(g.choice([20, 200, 2000]))
        for e in a:
            e.kind, e.count = int(g.choice([qb.QSV_S_F32, qb.QSV_S_BF16])), int(g.integers(0, 5))
            size = 4 if e.kind == qb.QSV_S_F32 else 2
            for name in ("param_dev", "m_dev", "v_dev"):
                at = 0x1000 + 4 * int(g.integers(0, wide))
                setattr(e, name, at)
                written += range(at, at + 4 * e.count)
            e.grad_dev = 0x1000 + size * int(g.integers(0, wide * 4 // size))
            read += range(e.grad_dev, e.grad_dev + size * e.count)
        fine = len(written) == len(set(written)) and not set(written) & set(read)
        assert (checks.request_adam(a, n, 1.0) is None) == fine, trial
        let += fine
    assert 400 < let < 3600


def test_norms_that_lie_in_a_tensor(checks):
    checks.request_clip_norm.restype = checks.request_adam_norm.restype = ctypes.c_char_p
    checks.request_clip_norm.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p]
    checks.request_adam_norm.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p]
    g, o = tensors((0x1000, 3, 5, 8), (0, 0, 4, 4)), tensors((0x2000, 3, 5, 5), (0, 0, 4, 4))
    rows = {0x1000 + 4 * (8 * r + c) for r in range(3) for c in range(5)}
    for at in range(0xff0, 0x1070):
        for norm in (1.0, INF):
            said = checks.request_clip_norm(g, None, 2, norm, at)
            assert (said is not None) == any(at < w + 4 and at + 4 > w for w in rows), hex(at)
    assert checks.request_clip_norm(g, o, 2, 1.0, 0x1ffc) is None and checks.request_clip_norm(g, o, 2, 1.0, 0x203c) is None
    assert b"norm" in checks.request_clip_norm(g, o, 2, 1.0, 0x2000) and b"norm" in checks.request_clip_norm(g, o, 2, 1.0, 0x2038)
    a = (qb.qsv_adam_tensor * 1)()
    a[0].kind, a[0].param_dev, a[0].grad_dev, a[0].m_dev, a[0].v_dev, a[0].count = qb.QSV_S_BF16, 0x1000, 0x2000, 0x3000, 0x4000, 10
    for at in (0x1000, 0x1024, 0x2000, 0x2010, 0x3024, 0x4000):
        assert b"norm" in checks.request_adam_norm(a, 1, 1.0, at)
    for at in (None, 0xffc, 0x1028, 0x2014, 0x3028, 0x4028):
        assert checks.request_adam_norm(a, 1, 1.0, at) is None


def test_lists_hold_the_memory_that_they_name():
    import torch
    x = torch.ones(1000)
    kept, at = (qb.TensorList([x]), qb.AdamList([x], [x], [x], [x])), x.data_ptr()
    x.data = torch.zeros(1000)
    assert x.data_ptr() != at and kept[0].at[0].data_dev == at and kept[1].at[0].param_dev == at
    assert len(kept[0].held) == 1 and len(kept[1].held) == 4 and all(s.data_ptr() == at for k in kept for s in k.held)


def test_lists_that_the_binding_refuses():
    import torch
    z = torch.zeros((4, 6))
    a = qb.TensorList([z, z[:, :5], z[1], torch.zeros((2, 3, 4)).half(), torch.zeros(()), torch.zeros((0, 3)), torch.zeros((5, 1))])
    assert [(e.rows, e.cols, e.row_stride) for e in a.at] == [(4, 6, 6), (4, 5, 6), (1, 6, 6), (1, 24, 24), (1, 1, 1), (0, 3, 3), (5, 1, 1)]
    assert len(a) == 7 and a.devices == {-1} and a.at[3].kind == qb.QSV_S_F16
    for bad in (z.t(), z[:, ::2], torch.zeros((2, 3, 4))[:, :, :2], z.double(), z.int(), z[:1].expand(4, 6)):
        with pytest.raises(qb.QsvError) as e:
            qb.TensorList([z, bad])
        assert e.value.status == qb.QSV_ERR_INVALID_ARG
    p = [torch.zeros(5) for _ in range(4)]
    assert qb.AdamList(*[[x] for x in p]).at[0].count == 5
    for lists in ([[p[0]], [p[1]], [p[2]], []], [[p[0].half()], [p[1]], [p[2]], [p[3]]], [[p[0]], [p[1].double()], [p[2]], [p[3]]],
                  [[p[0]], [p[1][:4]], [p[2]], [p[3]]], [[z[:, 0]], [z[:, 1]], [z[:, 2]], [z[:, 3]]]):
        with pytest.raises(qb.QsvError):
            qb.AdamList(*lists)


def test_layouts():
    assert [ctypes.sizeof(x) for x in (qb.qsv_tensor, qb.qsv_adam_tensor)] == [40, 48]


# ---- on the GPU ------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ctx():
    c = qb.Context(1, 1)
    yield c
    c.close()


def f64(t):
    return t.double().cpu().numpy()


def draw(shapes, seed, scale=0.1):
    """shapes: (type, rows, cols, padding); a vector has rows 0.  GPU tensors, rows of padded ones lie further apart."""
    import torch
    g = torch.Generator().manual_seed(seed)
    got = []
    for src, rows, cols, pad in shapes:
        x = (torch.randn((max(rows, 1), cols + pad), generator=g) * scale).to(tt(src)).cuda()
        got.append(x[:, :cols] if rows else x[0, :cols])
    return got


def norm_of(grads):
    return math.sqrt(math.fsum(float((f64(g) ** 2).sum()) for g in grads))


def check_clip(ctx, grads, most, over):
    import torch
    n, before = norm_of(grads), [f64(g) for g in grads]
    f = most / n if n > most else 1.0
    norm = torch.full((1,), 77.0, device="cuda")
    whole = [torch.full((g.shape[0], g.stride(0)) if g.dim() == 2 else g.shape, 55.0, dtype=g.dtype, device="cuda") for g in grads]
    outs = [w[:, :g.shape[1]] if g.dim() == 2 else w for w, g in zip(whole, grads)]
    if over:
        for o, g in zip(outs, grads):
            o.copy_(g)
        ctx.qsv_clip_grads(outs, most, norm=norm)
    else:
        ctx.qsv_clip_grads(qb.TensorList(grads), most, norm=norm, out=qb.TensorList(outs))
    torch.cuda.synchronize()
    assert abs(norm.item() - n) <= n * 1.5 * U
    for w, o, g, b in zip(whole, outs, grads, before):
        assert np.array_equal(f64(g), b)
        if g.dim() == 2:
            assert bool((w[:, g.shape[1]:] == 55.0).all())
        t = torch.finfo(g.dtype)
        half = np.maximum(t.eps / 2 * np.abs(b * f), t.smallest_normal * t.eps / 2)
        assert (np.abs(f64(o) - b * f) <= (half + U * np.abs(b * f)) * (1 + t.eps)).all()
    return norm


MIXED = [("f32", 10, 64, 0), ("f32", 0, 1, 0), ("bf16", 33, 65, 3), ("f16", 129, 7, 1), ("f32", 5, 1, 1), ("bf16", 0, 4099, 0), ("f16", 3, 9001, 5),
         ("f32", 2, 20011, 1), ("f32", 700, 12, 4), ("bf16", 1, 333, 8), ("f16", 64, 128, 0), ("f32", 0, 3, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("most", [0.0, 0.01, 1.0, 1e9, INF])
def test_mixed_tensors(ctx, most):
    grads = draw(MIXED, 1)
    for over in (False, True):
        check_clip(ctx, grads, most, over)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 255, 1000, 8191, 8193, 16384, 16385, 32769, 65537, 300001, 5000003])
def test_one_tensor(ctx, src, n):
    for over in (False, True):
        check_clip(ctx, draw([(src, 0, n, 0)], n), 0.5, over)
    x = draw([(src, 0, n + 3, 0)], n)[0]
    check_clip(ctx, [x[1:n + 1]], 0.25, False)                 # not aligned to a vector


@pytest.mark.gpu
@pytest.mark.parametrize("count", [57, 58, 59, 60, 61, 130, 200, 201, 700])
def test_long_lists(ctx, count):
    g = np.random.default_rng(count)
    shapes = [(("f32", "f16", "bf16")[int(g.integers(3))], int(g.integers(0, 20)), int(g.integers(0, 300)), int(g.integers(0, 3))) for _ in range(count)]
    grads = draw(shapes, count)
    for over in (False, True):
        check_clip(ctx, grads, 0.5, over)


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[("f32", 3001, 9001, 3), ("bf16", 0, 20000011, 0)] + MIXED, [("f16", 0, 1200001 + i, 0) for i in range(60)] + MIXED],
                         ids=["rows", "vectors"])
@pytest.mark.parametrize("most", [0.5, 1e9])
def test_results_past_the_caches(ctx, shapes, most):
    grads = draw(shapes, 9)
    for over in (False, True):
        check_clip(ctx, grads, most, over)


@pytest.mark.gpu
def test_many_rows_of_few_columns(ctx):
    for shape in (("f32", 300000, 1, 1), ("bf16", 100000, 5, 3), ("f16", 20000, 129, 7), ("f32", 4000, 4097, 3), ("f16", 3000, 4095, 1)):
        check_clip(ctx, draw([shape], 3), 0.5, False)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(7, 24), (300, 1031), (40, 9001)])
def test_tensors_of_one_buffer(ctx, src, rows, cols):
    """Columns, single rows between them and every other row of the rest, in place and into such places of another buffer: what lies between
    them is left as it is."""
    import torch
    a, b = cols // 3 - 1, cols // 2 + 1
    parts = lambda x: [x[:, :a], x[0, a:b], x[1::2, a:b], x[2::4, a:b], x[:, b + 1:cols - 1], x[rows - 1, cols - 1:]]  # noqa: E731
    buffer = draw([(src, rows, cols, 0)], rows)[0]
    grads, lone = parts(buffer), torch.ones_like(buffer, dtype=torch.bool)
    for x in parts(lone):
        x.fill_(False)
    n, before = norm_of(grads), f64(buffer)
    assert 0 < int(lone.sum()) < buffer.numel()
    norm, t = torch.zeros((1,), device="cuda"), torch.finfo(buffer.dtype)
    for most in (n / 2.5, 2 * n):
        f, other, over = min(1.0, most / n), torch.full_like(buffer, 55.0), buffer.clone()
        ctx.qsv_clip_grads(parts(buffer), most, norm=norm, out=parts(other))
        ctx.qsv_clip_grads(parts(over), most)
        assert abs(norm.item() - n) <= n * 1.5 * U and np.array_equal(f64(buffer), before)
        assert bool((other[lone] == 55.0).all()) and torch.equal(over[lone], buffer[lone]) and torch.equal(over[~lone], other[~lone])
        want = (before * f)[~lone.cpu().numpy()]
        half = np.maximum(t.eps / 2 * np.abs(want), t.smallest_normal * t.eps / 2)
        assert (np.abs(f64(over[~lone]) - want) <= (half + U * np.abs(want)) * (1 + t.eps)).all()


@pytest.mark.gpu
def test_empty_lists_and_tensors(ctx):
    import torch
    norm = torch.full((1,), 9.0, device="cuda")
    for grads in ([], [torch.zeros((0, 5), device="cuda")], [torch.zeros(70, device="cuda")]):
        for most in (1.0, INF):
            norm.fill_(9.0)
            ctx.qsv_clip_grads(grads, most, norm=norm)
            assert norm.item() == 0.0
    x = torch.zeros(70, device="cuda")
    ctx.qsv_clip_grads([x], 0.0)
    assert bool((x == 0).all())
    empty = [torch.zeros((0,), device="cuda")]
    norm.fill_(9.0)
    ctx.qsv_adam_clipped(qb.AdamList(empty, empty, empty, empty), 1, 0.1, 1.0, norm=norm)
    assert norm.item() == 0.0
    ctx.qsv_adam_clipped(qb.AdamList([], [], [], []), 1, 0.1, 1.0)


@pytest.mark.gpu
def test_sizes_of_values(ctx):
    """Squares beyond float32's range at both ends, infinities and NaN."""
    import torch
    norm = torch.zeros((1,), device="cuda")
    for value in (1e30, 3e38, 1e-30, 2.0 ** -149):
        x = torch.full((1000,), value, device="cuda")
        ctx.qsv_clip_grads([x], 1e-25, norm=norm)
        want = float(torch.full((1,), value)[0]) * math.sqrt(1000)
        # below 2^-126 float32's numbers lie 2^-149 apart, and rounding N misses by up to half of that: sqrt(1000) 2^-149 = 31.62 2^-149
        # becomes 32 2^-149, off by 0.38 2^-149, where 1.5 U of it would be 2.8e-6 2^-149
        assert abs(norm.item() - want) <= want * 1.5 * U + 2.0 ** -150 if want < 3.4e38 else norm.item() == INF
    x = torch.tensor([1.0, INF, -2.0], device="cuda")
    ctx.qsv_clip_grads([x], 1.0, norm=norm)
    assert norm.item() == INF and x[0] == 0 and x[2] == 0 and bool(x[1].isnan())
    y = [torch.tensor([1.0, NAN], device="cuda"), torch.ones(5, device="cuda")]
    ctx.qsv_clip_grads(y, INF, norm=norm)
    assert math.isnan(norm.item()) and bool((y[1] == 1).all()) and y[0][0] == 1
    ctx.qsv_clip_grads(y, 1.0, norm=norm)
    assert math.isnan(norm.item()) and bool(y[1].isnan().all()) and bool(y[0].isnan().all())


@pytest.mark.gpu
def test_the_same_bits_every_time(ctx):
    import torch
    grads, ref = draw(MIXED + [("f32", 0, 3000001, 0)], 6), None
    for _ in range(3):
        norm, outs = torch.zeros((1,), device="cuda"), [torch.zeros_like(g) for g in grads]
        ctx.qsv_clip_grads(grads, 0.3, norm=norm, out=outs)
        bits = [x.clone() for x in [norm] + outs]
        assert ref is None or all(torch.equal(a, b) for a, b in zip(ref, bits))
        ref = bits


def adam(p, g, m, v, f, t, lr, b1, b2, eps):
    g = g * f
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


def moments(grads, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    p = [torch.randn(x.shape, generator=g).cuda() for x in grads]
    m = [(torch.randn(x.shape, generator=g) * 0.03).cuda() for x in grads]
    v = [(torch.rand(x.shape, generator=g) * 0.01).cuda() for x in grads]
    return p, m, v


def check_adam(ctx, grads, most, t, lr=0.02, b1=0.9, b2=0.99, eps=1e-6, zero=False, seed=1):
    import torch
    p, m, v = moments(grads, seed)
    if zero:
        for x in m + v:
            x.zero_()
    n = norm_of(grads)
    f = most / n if n > most else 1.0
    want = [adam(*(f64(x) for x in y), f, t, lr, b1, b2, eps) for y in zip(p, grads, m, v)]
    first = [(f64(x), f64(y)) for x, y in zip(p, m)]
    norm = torch.full((1,), 77.0, device="cuda")
    ctx.qsv_adam_clipped(qb.AdamList(p, grads, m, v), t, lr, most, b1, b2, eps, norm=norm)
    torch.cuda.synchronize()
    assert abs(norm.item() - n) <= n * 1.5 * U
    for (wp, wm, wv), a, b, c, (p0, m0) in zip(want, p, m, v, first):
        tiny = 2.0 ** -149
        assert (np.abs(f64(b) - wm) <= U * np.abs(wm) + 2.0 ** -50 * np.abs(m0) + tiny).all()
        assert (np.abs(f64(c) - wv) <= U * np.abs(wv) * (1 + 2.0 ** -20) + tiny).all()
        assert (np.abs(f64(a) - wp) <= U * np.abs(wp) + 2.0 ** -48 * (np.abs(p0) + np.abs(wp - p0)) + tiny).all()


@pytest.mark.gpu
@pytest.mark.parametrize("most", [0.0, 0.05, 1e9, INF])
@pytest.mark.parametrize("t", [1, 7, 100000])
def test_adam_mixed(ctx, most, t):
    check_adam(ctx, draw([(s, r, c, 0) for s, r, c, _ in MIXED], 8), most, t, zero=t == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 255, 8191, 8193, 16385, 40001, 3000001])
def test_adam_one_tensor(ctx, src, n):
    check_adam(ctx, draw([(src, 0, n, 0)], n), 0.5, 3)
    x = draw([(src, 0, n + 3, 0)], n)[0]
    check_adam(ctx, [x[1:n + 1]], 0.25, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("most", [0.5, INF])
def test_adam_past_the_caches(ctx, most):
    shapes = [("f32", 0, 2000003, 0), ("bf16", 0, 2000001, 0), ("f16", 0, 1900003, 0), ("f32", 0, 7, 0)]
    check_adam(ctx, draw(shapes, 4), most, 3)
    check_adam(ctx, [x[1:] for x in draw(shapes, 5)], most, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [60, 61, 90, 91, 200, 201, 300])
def test_adam_long_lists(ctx, count):
    g = np.random.default_rng(count)
    check_adam(ctx, draw([(("f32", "f16", "bf16")[int(g.integers(3))], 0, int(g.integers(0, 4000)), 0) for _ in range(count)], count), 0.5, 4)


@pytest.mark.gpu
def test_adam_as_the_step_of_one_tensor(ctx):
    """Nothing to clip: bit for bit what qsv_adam_step gives."""
    import torch
    for n in (5, 320, 20001, 700001):
        g = draw([("f32", 0, n, 0)], n)[0]
        (p,), (m,), (v,) = moments([g], 2)
        a = [x.clone() for x in (p, m, v)]
        ctx.qsv_adam_step(p, g, m, v, 5, 0.01)
        ctx.qsv_adam_clipped(qb.AdamList([a[0]], [g], [a[1]], [a[2]]), 5, 0.01, INF)
        assert all(torch.equal(x, y) for x, y in zip((p, m, v), a))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_adam_leaves_a_step_out(ctx, bad):
    import torch
    for n in (50, 100000):
        grads = draw([("f32", 0, n, 0), ("bf16", 0, 77, 0)], 9)
        grads[0][n // 2] = bad
        p, m, v = moments(grads, 3)
        keep = [x.clone() for x in p + m + v]
        norm = torch.zeros((1,), device="cuda")
        for most in (1.0, INF):
            ctx.qsv_adam_clipped(qb.AdamList(p, grads, m, v), 3, 0.1, most, norm=norm)
            assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(bad)
            assert all(torch.equal(x, y) for x, y in zip(p + m + v, keep))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1000, 100000], ids=["one launch", "two launches"])
def test_adam_leaves_a_step_out_by_the_norm_that_it_reports(ctx, n):
    """Finite gradients of 3e38: their norm is finite in float64 and infinite in float32, which is what a program sees.  One of them alone has a
    norm of 3e38, and the step is taken."""
    import torch
    grads = [torch.full((n,), 3e38, device="cuda"), torch.zeros(77, dtype=torch.bfloat16, device="cuda")]
    p, m, v = moments(grads, 3)
    keep = [x.clone() for x in p + m + v]
    norm = torch.zeros((1,), device="cuda")
    for most in (1.0, INF):
        norm.zero_()
        ctx.qsv_adam_clipped(qb.AdamList(p, grads, m, v), 3, 0.1, most, norm=norm)
        assert norm.item() == INF and all(torch.equal(x, y) for x, y in zip(p + m + v, keep))
    grads[0][1:] = 0.0
    ctx.qsv_adam_clipped(qb.AdamList(p, grads, m, v), 3, 0.1, 1.0, norm=norm)
    assert norm.item() == grads[0][0].item() and not any(torch.equal(x, y) for x, y in zip(p + m + v, keep))


@pytest.mark.gpu
def test_refused_on_the_device(ctx):
    import torch
    x = torch.zeros(10, device="cuda")
    y = [torch.zeros(10, device="cuda") for _ in range(4)]
    for call in (lambda: ctx.qsv_clip_grads([x, x], 1.0), lambda: ctx.qsv_clip_grads([x.cpu()], 1.0), lambda: ctx.qsv_clip_grads([x], -1.0),
                 lambda: ctx.qsv_clip_grads([x], 1.0, out=[y[0], y[1]]), lambda: ctx.qsv_clip_grads([x], 1.0, out=[y[0][:5]]),
                 lambda: ctx.qsv_clip_grads([x], 1.0, norm=y[0]), lambda: ctx.qsv_adam_clipped([x], 1, 0.1, 1.0),
                 lambda: ctx.qsv_adam_clipped(qb.AdamList([x], [x], [y[0]], [y[1]]), 1, 0.1, 1.0),
                 lambda: ctx.qsv_adam_clipped(qb.AdamList(*[[t] for t in y]), 0, 0.1, 1.0),
                 lambda: ctx.qsv_adam_clipped(qb.AdamList(*[[t] for t in y]), 1, 0.1, 1.0, beta1=1.0),
                 lambda: ctx.qsv_adam_clipped(qb.AdamList(*[[t] for t in y]), 1, 0.1, 1.0, eps=0.0)):
        with pytest.raises(qb.QsvError) as e:
            call()
        assert e.value.status == qb.QSV_ERR_INVALID_ARG
    assert bool((x == 0).all())


@pytest.mark.gpu
def test_captured_steps_replay(ctx):
    import torch
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = qb.Context(1, 1)
        for shapes in ([("f32", 0, 320, 0), ("f32", 10, 64, 0)], [("bf16", 0, 400001, 0)] + [("f32", 0, 50 + i, 0) for i in range(70)]):
            grads = draw(shapes, 4)
            p, m, v = moments(grads, 5)
            first = [x.clone() for x in p + m + v]
            lists, norm = qb.AdamList(p, grads, m, v), torch.zeros((1,), device="cuda")
            outs = [torch.zeros_like(x) for x in grads]
            lists_in, lists_out = qb.TensorList(grads), qb.TensorList(outs)

            def step():
                c.qsv_adam_clipped(lists, 2, 0.01, 0.5, norm=norm)
                c.qsv_clip_grads(lists_in, 0.125, out=lists_out)
            step()
            want = [x.clone() for x in p + m + v + outs + [norm]]
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
            for _ in range(3):
                for x, y in zip(p + m + v, first):
                    x.copy_(y)
                for x in outs + [norm]:
                    x.fill_(9.0)
                graph.replay()
                stream.synchronize()
                assert all(torch.equal(x, y) for x, y in zip(p + m + v + outs + [norm], want))
        c.close()


@pytest.mark.gpu
def test_training_step_from_scores_to_parameters(ctx):
    """Rows of scores under a mask, a shared bias and penalties, their loss against a teacher, its gradient back to the scores and the bias,
    and a clipped step of both: against the formulas in 64 bits on the CPU."""
    import torch
    rows, cols, top = 24, 501, 7
    g = np.random.default_rng(11)
    z = g.standard_normal((rows, cols)).astype(np.float32) * 3
    bias = g.standard_normal(cols).astype(np.float32)
    prior = g.integers(0, cols, (rows, 12)).astype(np.int32)
    by = g.choice(np.float32([1.0, 1.25]), rows)
    masks = g.integers(0, 2 ** 32, (2, (cols + 31) // 32), dtype=np.uint32)
    masks[1] = 0
    of = (np.arange(rows) % 3 - 1).astype(np.int32)                  # none, mask 0, one that leaves nothing
    k = np.arange(cols)
    allowed = np.stack([np.ones(cols, bool) if i < 0 else (masks[i].astype(np.int64)[k // 32] >> (k % 32)) & 1 == 1 for i in of])
    idx = np.stack([np.resize(np.flatnonzero(a), top) if a.any() else np.full(top, -1) for a in allowed]).astype(np.int32)
    logits = g.standard_normal((rows, top)).astype(np.float32)
    cuda = lambda a: torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).cuda()  # noqa: E731
    zd, bd = cuda(z.copy()), cuda(bias.copy())
    more = dict(prior=cuda(prior), repetition=cuda(by), masks=cuda(masks), mask_of=cuda(of))
    out, dz, db, loss = torch.zeros_like(zd), torch.zeros_like(zd), torch.zeros_like(bd), torch.zeros(rows, device="cuda")
    ctx.qsv_adjust(qb.QSV_S_F32, zd, out, bias=bd, **more)
    ctx.qsv_distill(qb.QSV_S_F32, out, cuda(idx), cuda(logits), loss=loss, grad=dz)
    ctx.qsv_adjust_grad(qb.QSV_S_F32, dz, grad=dz, scores=zd, grad_bias=db, **more)
    m, v = [torch.zeros_like(x) for x in (zd, bd)], [torch.zeros_like(x) for x in (zd, bd)]
    norm = torch.zeros((1,), device="cuda")
    got = f64(dz), f64(db)
    ctx.qsv_adam_clipped(qb.AdamList([zd, bd], [dz, db], m, v), 1, 0.1, 0.5, norm=norm)
    torch.cuda.synchronize()
    # the formulas
    seen = np.zeros((rows, cols), bool)
    seen[np.arange(rows)[:, None], prior] = True
    z64 = z.astype(np.float64)
    slope = np.where(seen, np.where(z64 > 0, 1.0 / by[:, None], by[:, None]), 1.0)
    s = np.where(allowed, z64 * slope + bias, -INF)
    G = np.zeros((rows, cols))
    for r in range(rows):
        if not allowed[r].any():
            assert loss[r].item() == 0.0
            continue
        e = np.exp(s[r] - s[r].max())
        q = np.exp(logits[r].astype(np.float64))
        q /= q.sum()
        G[r] = e / e.sum()
        np.add.at(G[r], idx[r], -q)
    wz, wb = np.where(allowed, G, 0.0) * slope, np.where(allowed, G, 0.0).sum(0)
    # e: three roundings of an exponent below 40 and the exponential's, relative 130 U; the sum over 501 values; the factors: 1024 U in all
    assert np.abs(got[0] - wz).max() <= 1024 * U * np.abs(G).max() * 1.25
    assert np.abs(got[1] - wb).max() <= 1024 * U * np.abs(G).sum(0).max()
    n = math.sqrt((got[0] ** 2).sum() + (got[1] ** 2).sum())
    assert abs(norm.item() - n) <= 1.5 * U * n and n > 0.5
    for now, was, grad in ((f64(zd), z64, got[0]), (f64(bd), bias.astype(np.float64), got[1])):
        want, _, _ = adam(was, grad, 0.0, 0.0, 0.5 / n, 1, 0.1, 0.9, 0.999, 1e-8)
        assert (np.abs(now - want) <= U * np.abs(want) + 2.0 ** -40).all()
