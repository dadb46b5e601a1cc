"""Aggregation and its gradients over scores of fp32's ends: a position bias
whose masks are the type's lowest value makes such scores, and times a scale
above 1 they leave fp32's range where their differences, which are all that a
softmax takes, do not.  Against the 64-bit forms; the bar of the library's
aggregation and backward pass (tests/parity.py)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from tests.parity import assert_close
from workloads import small_params

pytestmark = pytest.mark.gpu
LOW = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


LAYERS = [  # tiled aggregation, single pixels, direct kernels; 16 to 64 lanes a neighbour and the scatter kernels
    dict(T=3, C=8, H=12, W=13, HD=2, wt=2, ps=3, k=5), dict(T=2, C=16, H=9, W=11, ps=1, k=9),
    dict(T=2, C=24, H=10, W=9, ps=1, k=6, dist_type=1, stride0=2), dict(T=2, C=40, H=9, W=8, ps=5, k=4, dist_type=1),
    dict(T=2, C=70, H=7, W=8, ps=3, k=5), dict(T=2, C=7, H=9, W=9, ps=2, k=100, ws=9, wt=1),
    dict(T=2, C=64, H=9, W=10, HD=4, ps=7, k=3),
]


def _scores(p, seed):
    """Rows of ordinary scores, rows masked in part, rows wholly masked (alike, and to several depths), infinite and NaN
    scores beside them."""
    g = torch.Generator().manual_seed(seed)
    shp = B.out_shape(p)
    d = torch.randn(shp, generator=g)
    bad = LOW if p["dist_type"] == 0 else -LOW
    kind = torch.randint(0, 5, shp[:-1], generator=g)[..., None].expand(shp)
    some = torch.rand(shp, generator=g) < 0.5
    d = torch.where((kind == 1) & some, torch.full_like(d, bad), d)
    d = torch.where(kind == 2, torch.full_like(d, bad), d)
    deep = torch.where(some, torch.full_like(d, bad), torch.full_like(d, bad / 2))
    d = torch.where(kind == 3, deep, d)
    d = torch.where((kind == 4) & some, torch.full_like(d, -bad), d)  # and the other end
    odd = torch.randint(0, 50, shp, generator=g)
    for j, val in enumerate((float("inf"), -float("inf"), float("nan"))):
        d = torch.where(odd == j, torch.full_like(d, val), d)
    inds = torch.empty(shp + (3,))
    inds[..., 0] = torch.randint(0, p["T"], shp, generator=g).float()
    inds[..., 1:] = 2.0 * torch.randn(shp + (2,), generator=g)
    return d, inds


@pytest.mark.parametrize("scale", [10.0, 1.0, 0.25, -3.0])
@pytest.mark.parametrize("kw", LAYERS, ids=range(len(LAYERS)))
def test_scores_of_the_ends(dev, kw, scale):
    p = small_params(**kw)
    d, inds = _scores(p, 5)
    g = torch.Generator().manual_seed(6)
    q, k, v, go = (torch.randn(B.video_shape(p), generator=g) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), generator=g)
    to = lambda x: x.to(dev)  # noqa: E731
    print("ends", p, scale, flush=True)
    dl = d.double().requires_grad_()
    want = R.aggregate(v.double(), dl, inds, p, scale)
    assert bool(want.isfinite().all())
    out = B.snls_aggregate(to(v), to(d), to(inds), p, scale)
    assert_close(out.cpu().numpy(), want.detach().numpy(), "out")
    static = B.snls_aggregate_static(to(v), to(d), to(inds), p, scale)
    assert torch.equal(static, out)
    kept = B.snls_aggregate_stacked(to(v), to(d), to(inds), p, scale)  # (B, HD, k, T, Ch, H, W)
    kept = kept.sum(2).permute(0, 2, 1, 3, 4, 5).reshape(out.shape)
    assert_close(kept.cpu().numpy(), want.detach().numpy(), "stacked")
    ds, = torch.autograd.grad((want * go.double()).sum(), dl)
    got = B.snls_backward_scores(*(to(x) for x in (q, k, v, fl, d, inds, go)), p, scale)
    assert_close(got[4].cpu().numpy(), ds.numpy(), "grad_scores")
    ref = oracle.backward(*(x.numpy() for x in (q, k, v, fl, d, inds, go)), p, scale)
    for x, r, name in zip(got, ref, ("grad_q", "grad_k", "grad_v", "grad_flows")):
        assert_close(x.cpu().numpy(), r, name)


def test_mask_of_the_lowest_value_through_a_layer(dev):
    """A table that masks every displacement of a head, and another that masks a frame step, at the scale of 10 that the
    softmax of a layer takes: no NaN, a wholly masked row is the softmax of what is left beside the mask."""
    p, bias = small_params(T=3, C=16, H=14, W=15, HD=2, ws=3, wt=1, ps=1, k=6), dict(radius=1, edges=[0.5, 2.0])
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(B.video_shape(p), generator=g).to(dev) for _ in range(3))
    fl = torch.randn(B.flow_shape(p), generator=g).to(dev)
    table = torch.randn(B.bias_table_shape(bias, 2), generator=g)
    table[0] = LOW
    table[1, 0] = LOW
    d, i = B.snls_search(q, k, fl, p)
    db = B.snls_bias(d, i, table.to(dev), p, bias)
    out = B.snls_aggregate(v, db, i, p, 10.0)
    want = R.aggregate(v.cpu().double(), db.cpu().double(), i.cpu(), p, 10.0)
    assert bool(out.isfinite().all())
    assert_close(out.cpu().numpy(), want.numpy(), "out")
    go = torch.ones_like(v)
    for x in B.snls_backward_scores(q, k, v, fl, db, i, go, p, 10.0):
        assert bool(x.isfinite().all())
