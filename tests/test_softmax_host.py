"""Softmax attention's host side: buckets by integers, and what the entry points refuse (on a pretended device: no kernel runs)."""
import ctypes as C

import numpy as np
import pytest

from tests import fake_device
from tests import softmax_reference as R


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return fake_device.build(tmp_path_factory.mktemp("fake"))


@pytest.fixture
def fake(so):
    return fake_device.Fake(so)


@pytest.mark.parametrize("n,far", [(2, 2), (2, 1 << 24), (3, 2), (8, 5), (32, 128), (32, 129), (33, 1000), (63, 40), (64, 1 << 24), (64, 33)])
def test_buckets_by_integers(n, far):
    from paper_2410_03462_b200 import binding as B
    h, L = n // 2, n - n // 2
    want = list(range(h))
    for y in range(L):
        x = h
        lo, hi = h, far
        while lo < hi:
            x = (lo + hi) // 2
            if x ** L >= far ** y * h ** (L - y):
                hi = x
            else:
                lo = x + 1
        want.append(max(lo, want[-1] + 1))
    got = B.grf_relative_buckets(n, far)
    assert got.tolist() == want
    # borders: the distance itself is in its bucket, the one before is not
    d = np.array(want)
    assert (R.bucket(got, -d, False) == np.arange(n)).all() and (R.bucket(got, -(d[1:] - 1), False) == np.arange(n - 1)).all()


@pytest.mark.parametrize("n,far", [(1, 10), (65, 100), (32, 16), (8, 4), (8, (1 << 24) + 1), (0, 5), (-1, 5)])
def test_buckets_refused(n, far):
    from paper_2410_03462_b200 import binding as B
    with pytest.raises(B.GrfError) as e:
        B.grf_relative_buckets(n, far)
    assert e.value.code == B.GRF_ERR_INVALID


def _desc(**fields):
    from paper_2410_03462_b200 import binding as B
    s = B.SoftmaxDesc()
    for name, value in dict(dict(batch=2, heads=4, kv_heads=2, n_q=100, n_k=120, dim=64, dtype=1, scale=0.125), **fields).items():
        if name.endswith("_stride") or name == "first":
            getattr(s, name)[:len(value)] = value
        else:
            setattr(s, name, value)
    return s


SOME = 4096


def _call(fake, ctx, s, backward=False, ws=None, q=SOME, dtable=None, rest=None):
    p = lambda x: C.c_void_p(x)  # noqa: E731
    fn = fake.lib.grf_softmax_attn_workspace_bytes
    fn.restype, fn.argtypes = C.c_size_t, [C.c_void_p, C.c_void_p, C.c_int]
    need = fn(ctx, C.byref(s), int(backward)) if ws is None else ws
    if backward:
        return fake.lib.grf_softmax_attn_backward(ctx, C.byref(s), p(q), p(SOME), p(SOME), p(SOME), p(SOME), p(rest), p(SOME), p(SOME), p(SOME), p(SOME),
                                                  p(dtable), p(SOME), C.c_size_t(need))
    return fake.lib.grf_softmax_attn(ctx, C.byref(s), p(q), p(SOME), p(SOME), p(SOME), None, p(rest), p(SOME), C.c_size_t(need))


BUCKETS = dict(bias=2, n_buckets=3, first=[0, 1, 5], table=SOME)


@pytest.mark.parametrize("fields", [
    dict(), dict(order=1), dict(order=2, prefix=SOME), dict(bias=1, slopes=SOME), BUCKETS, dict(BUCKETS, two_sided=1), dict(q_doc=SOME, k_doc=SOME),
    dict(n_q=1), dict(n_q=16, n_k=1), dict(cap=3.0), dict(dtype=0, dim=8), dict(q_stride=[0, 64, 0]), dict(k_stride=[8, 0, 64]),
    dict(batch=1, out_stride=[3, 64, 256]), dict(out_stride=[64, 128, 1024]), dict(n_q=1 << 22, n_k=1 << 22)], ids=str)
def test_calls_that_are_taken(fake, fields):
    ctx = fake.context()
    s = _desc(**fields)
    for backward in (False, True):
        assert _call(fake, ctx, s, backward, dtable=SOME if "table" in fields and backward else None) == 0
    assert fake.launched("softmax") >= 2 and fake.errors() == 0


@pytest.mark.parametrize("fields,code", [
    (dict(batch=0), -1), (dict(heads=3), -1), (dict(kv_heads=0), -1), (dict(n_q=0), -1), (dict(n_k=-1), -1), (dict(dim=0), -1), (dict(dim=4), -1),
    (dict(dim=136), -1), (dict(dtype=2), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(cap=-1.0), -1), (dict(cap=float("inf")), -1),
    (dict(order=3), -1), (dict(order=-1), -1), (dict(order=2), -1), (dict(prefix=SOME), -1), (dict(bias=3), -1), (dict(bias=1), -1), (dict(slopes=SOME), -1),
    (dict(bias=2), -1), (dict(BUCKETS, n_buckets=0), -1), (dict(BUCKETS, n_buckets=65), -1), (dict(BUCKETS, first=[1, 2, 5]), -1),
    (dict(BUCKETS, first=[0, 5, 5]), -1), (dict(BUCKETS, first=[0, 5, (1 << 29) + 1]), -1), (dict(BUCKETS, two_sided=2), -1), (dict(q_doc=SOME), -1), (dict(k_doc=SOME), -1),
    (dict(q_stride=[4, 64, 64]), -1), (dict(q_stride=[64, 64, -64]), -1), (dict(k_stride=[1 << 37, 64, 64]), -1), (dict(out_stride=[25600, 0, 64]), -1),
    (dict(out_stride=[25600, 6400, 56]), -1), (dict(out_stride=[6400, 6400, 64]), -1), (dict(out_stride=[64, 64, 128]), -1),
    (dict(n_q=(1 << 22) + 1), -2), (dict(n_k=(1 << 22) + 1), -2), (dict(batch=40000), -2)], ids=str)
def test_calls_that_are_refused(fake, fields, code):
    ctx = fake.context()
    s = _desc(**fields)
    assert _call(fake, ctx, s) == code and _call(fake, ctx, s, ws=1 << 40) == code
    assert _call(fake, ctx, s, True, ws=1 << 40) == code
    fn = fake.lib.grf_softmax_attn_workspace_bytes
    assert fn(ctx, C.byref(s), 0) == 0 and fn(ctx, C.byref(s), 1) == 0
    assert fake.launched("softmax") == 0


def test_addresses_and_workspaces(fake):
    ctx = fake.context()
    s = _desc(q_doc=SOME, k_doc=SOME)
    fn = fake.lib.grf_softmax_attn_workspace_bytes
    fn.restype, fn.argtypes = C.c_size_t, [C.c_void_p, C.c_void_p, C.c_int]
    for backward in (False, True):
        need = fn(ctx, C.byref(s), int(backward))
        assert need > 0 and need % 256 == 0
        assert _call(fake, ctx, s, backward, ws=need - 1) == -3 and _call(fake, ctx, s, backward, ws=need) == 0
        assert _call(fake, ctx, s, backward, q=SOME + 8) == -1 and _call(fake, ctx, s, backward, q=None) == -1
        assert _call(fake, ctx, s, backward, rest=SOME) == 0 and _call(fake, ctx, s, backward, rest=SOME + 8) == -1
        assert _call(fake, ctx, _desc(dtype=0), backward, rest=SOME) == -1  # fp32 outputs are not rounded
    assert _call(fake, ctx, s, True, dtable=SOME) == -1                     # no table to have a gradient
    for stride in ("dq", "dk", "dv"):
        assert _call(fake, ctx, _desc(**{stride + "_stride": [6400, 0, 64]}), True) == -1, stride
    assert _call(fake, ctx, _desc(dout_stride=[0, 0, 64]), True) == 0
    # a long cache of one sequence: parts in the workspace
    long = _desc(batch=1, heads=1, kv_heads=1, n_q=1, n_k=200000)
    assert fn(ctx, C.byref(long), 0) > 0 and _call(fake, ctx, long) == 0 and fake.launched("few_join") == 1


def test_bias_calls(fake):
    ctx = fake.context()
    p = lambda x: C.c_void_p(x)  # noqa: E731
    first = np.array([0, 1, 4], np.int32)
    f = first.ctypes.data_as(C.c_void_p)
    wsb = fake.lib.grf_relative_bias_workspace_bytes
    wsb.restype = C.c_size_t
    rows = lambda *a: fake.lib.grf_relative_bias(ctx, *a)  # noqa: E731
    assert rows(4, 100, 100, 0, 3, 1, f, 1, p(SOME), p(SOME)) == 0
    for a in ((0, 100, 100, 0, 3, 1, f, 1, p(SOME), p(SOME)), (4, 0, 100, 0, 3, 1, f, 1, p(SOME), p(SOME)), (4, 100, 100, 0, 0, 1, f, 1, p(SOME), p(SOME)),
              (4, 100, 100, 0, 65, 1, f, 1, p(SOME), p(SOME)), (4, 100, 100, 0, 3, 2, f, 1, p(SOME), p(SOME)), (4, 100, 100, 0, 3, 1, None, 1, p(SOME), p(SOME)),
              (4, 100, 100, 0, 3, 1, f, 3, p(SOME), p(SOME)), (4, 100, 100, 0, 3, 1, f, 1, None, p(SOME)), (4, 100, 100, 0, 3, 1, f, 1, p(SOME), p(SOME + 2))):
        assert rows(*a) == -1
    assert rows(4, (1 << 22) + 1, 100, 0, 3, 1, f, 1, p(SOME), p(SOME)) == -2 and rows(65536, 1, 1, 0, 3, 1, f, 1, p(SOME), p(SOME)) == -2
    need = wsb(4, 100, 100, 3, 1)
    back = lambda batch, ws, n, drows=SOME: fake.lib.grf_relative_bias_backward(  # noqa: E731
        ctx, batch, 4, 100, 100, 0, 3, 1, f, 0, p(drows), p(SOME), p(ws), C.c_size_t(n))
    assert back(2, SOME, need) == 0
    assert back(0, SOME, need) == -1 and back(2, None, need) == -1 and back(2, SOME, need - 1) == -3 and back(2, SOME, need, SOME + 4) == -1
    assert fake.errors() == 0


def test_numbers_that_do_not_fit_are_refused_not_cut_off():
    import torch

    from paper_2410_03462_b200 import api
    from paper_2410_03462_b200 import binding as B
    assert list(B._distances([0, 1, 1 << 29])) == list(B._distances(np.array([0, 1, 1 << 29]))) == [0, 1, 1 << 29]
    for first in ([0, (1 << 32) + 1], [0, -(1 << 32) + 1], np.array([0, (1 << 32) + 1]), [0, 1.5]):
        with pytest.raises(ValueError):
            B._distances(first)

    class Some:
        device, torch_device, handle = 0, torch.device("cuda", 0), None

    class OnDevice:
        is_cuda = True

        def get_device(self):
            return 0
    for n_q, n_k, start in ((4, 4, 1 << 31), (4, 4, -(1 << 31) - 1), ((1 << 32) + 4, 4, 0), (4, (1 << 32) + 4, 0)):
        with pytest.raises(ValueError, match="32-bit"):
            api._first_position(Some, OnDevice(), n_q, n_k, start)
    assert api._first_position(Some, OnDevice(), 3, 7, None) == 4
    other = OnDevice()
    other.get_device = lambda: 1
    for t in (torch.zeros(2, 8), other):
        with pytest.raises(ValueError, match="cuda:0"):
            api._first_position(Some, t, 4, 4, 0)
    small = torch.zeros(1, 1, 1, 8)
    many = small.expand(1, 1, (1 << 32) + 4, 8)
    for q, k in ((many, small), (small, many)):
        with pytest.raises(ValueError, match="too many tokens"):
            api.softmax_attn(Some, q, k, k)


@pytest.mark.parametrize("fields", [dict(scale=3e38), dict(scale=-3e38), dict(cap=3e38), dict(cap=1e-40), dict(cap=1.0, scale=2.5e38), dict(cap=0.5, scale=2e38)], ids=str)
def test_scales_and_caps_that_overflow_are_refused(fake, fields):
    ctx = fake.context()
    s = _desc(**fields)
    assert _call(fake, ctx, s, ws=1 << 40) == -1 and _call(fake, ctx, s, True, ws=1 << 40) == -1
    assert fake.launched("softmax") == 0


@pytest.mark.parametrize("fields", [dict(scale=2e38), dict(cap=2e38), dict(cap=1e-37), dict(cap=1.0, scale=2e38), dict(cap=1e-40, scale=0.0)], ids=str)
def test_scales_and_caps_that_do_not_overflow_are_taken(fake, fields):
    ctx = fake.context()
    assert _call(fake, ctx, _desc(**fields)) == 0 and _call(fake, ctx, _desc(**fields), True) == 0


def test_calls_too_large_are_told_so_without_a_workspace(fake):
    """A size of 0 is what a caller gets for them, so there is no workspace to bring."""
    ctx = fake.context()
    p = lambda x: C.c_void_p(x)  # noqa: E731
    s = _desc(batch=40000)
    fn = fake.lib.grf_softmax_attn_backward
    assert fn(ctx, C.byref(s), *(p(x) for x in (SOME,) * 5), None, *(p(x) for x in (SOME,) * 4), None, None, C.c_size_t(0)) == -2
    assert fn(ctx, C.byref(_desc()), *(p(x) for x in (SOME,) * 5), None, *(p(x) for x in (SOME,) * 4), None, None, C.c_size_t(0)) == -1
    first = np.array([0, 1, 4], np.int32).ctypes.data_as(C.c_void_p)
    assert fake.lib.grf_relative_bias_backward(ctx, 1, 65536, 1, 1, 0, 3, 1, first, 0, p(SOME), p(SOME), None, C.c_size_t(0)) == -2
    assert fake.lib.grf_relative_bias_backward(ctx, 1, 4, 1, 1, 0, 3, 1, first, 0, p(SOME), p(SOME), None, C.c_size_t(0)) == -1


def test_masks_that_there_are_not():
    import torch

    from paper_2410_03462_b200 import api
    x = torch.zeros(1, 1, 1, 8)
    for mask in ("casual", None, "PREFIX"):
        with pytest.raises(ValueError, match="full, causal, prefix"):
            api.softmax_attn(None, x, x, x, mask=mask)
