"""Refusals of the position bias and of the 8-bit frame cache (before any
buffer or the device is touched), and checks of their plain 64-bit forms."""
import ctypes
import math

import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import attention64 as R

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def _params(**kw):
    p = dict(B=1, T=3, C=8, H=16, W=17, HD=2, ws=3, wt=1, ps=3, stride0=1, stride1=1.0, k=4, dist_type=0)
    p.update(kw)
    return B.params_from_dict(p)


def _bias(radius=1, edges=(0.5, 2.0)):
    return B.bias_from_dict(dict(radius=radius, edges=list(edges)))


def _cache(**kw):
    c = dict(B=1, slots=3, C=32, H=16, W=17, HD=2, block=8)
    c.update(kw)
    return B.cache_from_dict(c)


def test_struct_sizes():
    assert ctypes.sizeof(B.SnlsBiasParams) == 4 * (3 + B.SNLS_BIAS_MAX_EDGES)
    assert ctypes.sizeof(B.SnlsCacheParams) == 4 * 8


BAD_BIAS = [
    (_bias(radius=-1), B.SNLS_ERR_INVALID_ARG), (_bias(radius=64, edges=()), B.SNLS_ERR_UNSUPPORTED),
    (_bias(edges=(1.0, 1.0)), B.SNLS_ERR_INVALID_ARG), (_bias(edges=(2.0, 1.0)), B.SNLS_ERR_INVALID_ARG),
    (_bias(edges=(0.0, 1.0)), B.SNLS_ERR_INVALID_ARG), (_bias(edges=(-1.0,)), B.SNLS_ERR_INVALID_ARG),
    (_bias(edges=(1.0, math.inf)), B.SNLS_ERR_INVALID_ARG), (_bias(edges=(math.nan,)), B.SNLS_ERR_INVALID_ARG),
    (_bias(edges=[float(i + 1) for i in range(17)]), B.SNLS_ERR_UNSUPPORTED),
    (_bias(radius=2, edges=[float(i + 1) for i in range(15)]), B.SNLS_ERR_UNSUPPORTED),  # 5 * 31^2 buckets
]


@pytest.mark.parametrize("bias,want", BAD_BIAS, ids=range(len(BAD_BIAS)))
def test_bias_refuses_bad_buckets(lib, bias, want):
    prm, cp = _params(), _cache()
    bp = ctypes.byref(bias)
    assert lib.snls_bias(FAKE, FAKE, FAKE, ctypes.byref(prm), bp, FAKE, None) == want
    assert lib.snls_bias_backward(FAKE, FAKE, FAKE, ctypes.byref(prm), bp, FAKE, FAKE, BIG, None) == want
    assert lib.snls_cache_attend(*[FAKE] * 8, ctypes.byref(cp), bp, 3, 1.0, FAKE, None) == want


def test_bias_refuses_bad_arguments(lib):
    prm, bias = _params(), _bias()
    pp, bp = ctypes.byref(prm), ctypes.byref(bias)
    for i in range(4):
        a = [FAKE] * 4
        a[i] = None
        assert lib.snls_bias(a[0], a[1], a[2], pp, bp, a[3], None) == B.SNLS_ERR_INVALID_ARG
        assert lib.snls_bias_backward(a[0], a[1], a[2], pp, bp, a[3], FAKE, BIG, None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_bias(FAKE, FAKE, FAKE, pp, None, FAKE, None) == B.SNLS_ERR_INVALID_ARG
    bad = _bias()
    bad.struct_size = 8
    assert lib.snls_bias(FAKE, FAKE, FAKE, pp, ctypes.byref(bad), FAKE, None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_bias(FAKE, FAKE, FAKE, ctypes.byref(_params(ws=0)), bp, FAKE, None) == B.SNLS_ERR_INVALID_ARG
    need = lib.snls_workspace_size(B.SNLS_OP_BIAS_BACKWARD, pp)
    assert 0 < need < 1 << 30
    assert lib.snls_workspace_size(B.SNLS_OP_BIAS_BACKWARD, ctypes.byref(_params(k=0))) != ctypes.c_size_t(-1).value
    assert lib.snls_workspace_size(B.SNLS_OP_BIAS_BACKWARD, ctypes.byref(_params(ws=0))) == ctypes.c_size_t(-1).value
    for ws, n in ((None, BIG), (FAKE, need - 1), (ctypes.c_void_p(0x1104), BIG)):
        assert lib.snls_bias_backward(FAKE, FAKE, FAKE, pp, bp, FAKE, ws, n, None) == B.SNLS_ERR_WORKSPACE


def test_backward_scores_refuses(lib):
    pp = ctypes.byref(_params())
    need = lib.snls_workspace_size(B.SNLS_OP_BACKWARD, pp)
    grads = [FAKE] * 5
    for i in range(5):
        g = list(grads)
        g[i] = None
        assert lib.snls_backward_scores(*[FAKE] * 8, pp, 1.0, *g, FAKE, BIG, None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_backward_scores(*[FAKE] * 8, pp, 1.0, *grads, FAKE, need - 1, None) == B.SNLS_ERR_WORKSPACE
    assert lib.snls_backward_scores(*[FAKE] * 8, pp, math.nan, *grads, FAKE, BIG, None) == B.SNLS_ERR_INVALID_ARG


BAD_CACHE = [
    (dict(B=0), B.SNLS_ERR_INVALID_ARG), (dict(slots=0), B.SNLS_ERR_INVALID_ARG), (dict(C=33), B.SNLS_ERR_INVALID_ARG),
    (dict(H=0), B.SNLS_ERR_INVALID_ARG), (dict(W=-1), B.SNLS_ERR_INVALID_ARG), (dict(block=0), B.SNLS_ERR_INVALID_ARG),
    (dict(block=4), B.SNLS_ERR_UNSUPPORTED), (dict(block=32), B.SNLS_ERR_UNSUPPORTED),
    (dict(C=514), B.SNLS_ERR_UNSUPPORTED), (dict(H=1000000, W=1), B.SNLS_ERR_UNSUPPORTED),
    (dict(H=40000, W=40000), B.SNLS_ERR_UNSUPPORTED),  # a plane of 2^31 bytes or more
    (dict(B=1 << 20, H=1 << 10, W=1 << 10), B.SNLS_ERR_UNSUPPORTED),
    (dict(B=1 << 10, H=1 << 9, W=1 << 10), B.SNLS_ERR_UNSUPPORTED),  # 2^30 pixels and heads
    (dict(B=1 << 20, H=3, W=3), B.SNLS_ERR_UNSUPPORTED),  # ... of padded frames
    (dict(B=1 << 16, slots=1 << 15, H=3, W=3), B.SNLS_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("kw,want", BAD_CACHE, ids=[str(k) for k, _ in BAD_CACHE])
def test_cache_refuses_bad_sizes(lib, kw, want):
    cp = ctypes.byref(_cache(**kw))
    assert lib.snls_cache_store(FAKE, FAKE, FAKE, cp, FAKE, FAKE, FAKE, FAKE, None) == want
    assert lib.snls_cache_attend(*[FAKE] * 7, None, cp, None, 3, 1.0, FAKE, None) == want
    assert lib.snls_cache_attend_points(FAKE, FAKE, 5, *[FAKE] * 6, None, cp, None, 3, 1.0, FAKE,
                                        None) == want


def test_cache_refuses_bad_arguments(lib):
    cp, odd = ctypes.byref(_cache()), ctypes.c_void_p(0x1008)
    bias = ctypes.byref(_bias())
    for i in range(7):
        a = [FAKE] * 7
        a[i] = None
        assert lib.snls_cache_store(*a[:3], cp, *a[3:], None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_cache_store(FAKE, FAKE, FAKE, cp, odd, FAKE, FAKE, FAKE, None) == B.SNLS_ERR_INVALID_ARG
    for i in (0, 2, 3, 4, 5, 6):  # flows (1) may be NULL
        a = [FAKE] * 7
        a[i] = None
        assert lib.snls_cache_attend(*a, None, cp, None, 3, 1.0, FAKE, None) == B.SNLS_ERR_INVALID_ARG
        assert lib.snls_cache_attend_points(a[0], FAKE, 5, *a[1:], None, cp, None, 3, 1.0, FAKE,
                                            None) == B.SNLS_ERR_INVALID_ARG
    ok = [FAKE] * 7
    bad = _cache()
    bad.struct_size = 4
    for args, want in (((None, cp, bias, 3, 1.0, FAKE), B.SNLS_ERR_INVALID_ARG),  # bias without a table
                       ((FAKE, cp, None, 3, 1.0, FAKE), B.SNLS_ERR_INVALID_ARG),  # ... and a table without
                       ((None, cp, None, 0, 1.0, FAKE), B.SNLS_ERR_INVALID_ARG),
                       ((None, cp, None, 16, 1.0, FAKE), B.SNLS_ERR_UNSUPPORTED),
                       ((None, cp, None, 3, math.inf, FAKE), B.SNLS_ERR_INVALID_ARG),
                       ((None, cp, None, 3, 1.0, None), B.SNLS_ERR_INVALID_ARG),
                       ((None, None, None, 3, 1.0, FAKE), B.SNLS_ERR_INVALID_ARG),
                       ((None, ctypes.byref(bad), None, 3, 1.0, FAKE), B.SNLS_ERR_INVALID_ARG)):
        assert lib.snls_cache_attend(*ok, *args, None) == want
        assert lib.snls_cache_attend_points(FAKE, FAKE, 5, *ok[1:], *args, None) == want
    assert lib.snls_cache_attend(FAKE, FAKE, FAKE, odd, *[FAKE] * 3, None, cp, None, 3, 1.0, FAKE,
                                 None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_cache_attend_points(FAKE, None, 5, *ok[1:], None, cp, None, 3, 1.0, FAKE,
                                        None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_cache_attend_points(FAKE, FAKE, -1, *ok[1:], None, cp, None, 3, 1.0, FAKE,
                                        None) == B.SNLS_ERR_INVALID_ARG
    assert lib.snls_cache_attend_points(FAKE, FAKE, 1 << 30, *ok[1:], None, cp, None, 3, 1.0, FAKE,
                                        None) == B.SNLS_ERR_UNSUPPORTED
    assert lib.snls_cache_attend_points(FAKE, FAKE, (1 << 29) - 64, *ok[1:], None, cp, None, 3, 1.0, FAKE,
                                        None) == B.SNLS_ERR_UNSUPPORTED  # a launch of 2^32 threads
    assert lib.snls_cache_attend_points(FAKE, FAKE, 0, *ok[1:], None, cp, None, 3, 1.0, FAKE, None) == B.SNLS_OK


def test_bias_refuses_too_many(lib):
    bp = ctypes.byref(_bias())
    many = ctypes.byref(_params(B=1 << 13, T=1 << 10, H=16, W=16))  # 2^24 images
    long = ctypes.byref(_params(B=1 << 10, T=1 << 10, H=1 << 10, W=1 << 10, k=1))  # 2^41 scores
    heads = ctypes.byref(_params(B=1, T=1, C=1 << 17, HD=1 << 16, H=16, W=16))
    for pp in (many, long):
        assert lib.snls_bias(FAKE, FAKE, FAKE, pp, bp, FAKE, None) == B.SNLS_ERR_UNSUPPORTED
        assert lib.snls_bias_backward(FAKE, FAKE, FAKE, pp, bp, FAKE, FAKE, BIG, None) == B.SNLS_ERR_UNSUPPORTED
    assert lib.snls_bias_backward(FAKE, FAKE, FAKE, heads, bp, FAKE, FAKE, BIG, None) == B.SNLS_ERR_UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device error path")
def test_valid_calls_without_device(lib):
    prm, bias, cp = ctypes.byref(_params()), ctypes.byref(_bias()), ctypes.byref(_cache())
    assert lib.snls_bias(FAKE, FAKE, FAKE, prm, bias, FAKE, None) == B.SNLS_ERR_HIP
    assert lib.snls_bias_backward(FAKE, FAKE, FAKE, prm, bias, FAKE, FAKE, BIG, None) == B.SNLS_ERR_HIP
    assert lib.snls_cache_store(FAKE, FAKE, FAKE, cp, FAKE, FAKE, FAKE, FAKE, None) == B.SNLS_ERR_HIP
    assert lib.snls_cache_attend(*[FAKE] * 8, cp, bias, 15, 1.0, FAKE, None) == B.SNLS_ERR_HIP


def test_binding_refuses_cpu_tensors_and_shapes():
    cp = dict(B=1, slots=1, C=4, H=4, W=4, HD=1, block=8)
    cache = B.cache_alloc(cp, "cpu")
    assert cache[0].shape == (1, 1, 1, 4, 4, 16) and cache[1].shape == (1, 1, 1, 1, 1)
    with pytest.raises(ValueError):
        B.snls_cache_attend(torch.zeros(1, 4, 4, 4), None, torch.zeros(1, 1, dtype=torch.int32), cache, cp, 3)
    p = dict(B=1, T=1, C=2, H=4, W=4, HD=1, ws=3, wt=0, ps=1, stride0=1, stride1=1.0, k=2, dist_type=0)
    with pytest.raises(ValueError):
        B.snls_bias(torch.zeros(1, 1, 1, 4, 4, 2), torch.zeros(1, 1, 1, 4, 4, 2, 3), torch.zeros(1, 1, 1, 1), p,
                    dict(radius=0, edges=[]))


def test_plain_rounding_is_e4m3():
    """The 64-bit rounding agrees with torch's conversion on every half-way point and neighbour of e4m3."""
    vals = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()  # 0 .. 448, ascending
    mid = (vals[1:] + vals[:-1]) / 2
    x = torch.cat([vals, mid, torch.nextafter(mid, mid + 1), torch.nextafter(mid, mid - 1)])
    x = torch.cat([x, -x, torch.tensor([448.0])])
    codes, scales = R.e4m3(x.view(1, 1, -1, 1, 1), 8)
    assert float(scales) == 1.0
    assert torch.equal(codes.flatten().float(), x.to(torch.float8_e4m3fn).float())


def test_plain_table_gradient_is_the_differences():
    """table_grad against central differences of a loss through the bias, the softmax and the aggregation."""
    torch.manual_seed(0)
    for dist in (0, 1):
        p = dict(B=1, T=2, C=4, H=5, W=6, HD=2, ws=3, wt=1, ps=3, stride0=2, stride1=1.0, k=3, dist_type=dist)
        bias = dict(radius=1, edges=[0.75, 2.0])
        shp = B.out_shape(p)
        inds = torch.cat([torch.randint(0, 2, shp + (1,)).float(), 2.5 * torch.randn(shp + (2,))], -1)
        d = torch.randn(shp, dtype=R.F64)
        d[0, 0, 0, 0, 0] = math.inf if dist else -math.inf
        table, v, go = (torch.randn(s, dtype=R.F64) for s in ((2, 3, 5, 5), (1, 2, 4, 5, 6), (1, 2, 4, 5, 6)))

        def loss(tb):
            return (R.aggregate(v, R.biased(d, inds, tb, p, bias), inds, p, 0.7) * go).sum()

        db = R.biased(d, inds, table, p, bias).requires_grad_()
        g, = torch.autograd.grad((R.aggregate(v, db, inds, p, 0.7) * go).sum(), db)
        got, _, _ = R.table_grad(g, d, inds, p, bias, 2)
        for at in ((0, 1, 2, 2), (1, 0, 3, 1), (0, 2, 0, 4), (1, 1, 2, 3)):
            e = torch.zeros_like(table)
            e[at] = 1e-5
            num = float(loss(table + e) - loss(table - e)) / 2e-5
            assert abs(num - float(got[at])) <= 1e-7 * max(1.0, abs(num)), (dist, at)
