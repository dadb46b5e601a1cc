"""Gradients of rows with finite scores at positions that are not read (frame
outside the clip or not whole, displacement far or not finite).

Such a neighbour brings nothing to the sum, but its score stays in the softmax
(include/snls.h, snls_aggregate): it scales every other weight, so the loss
depends on it.  The bar is that of the library's backward pass
(tests/parity.py): fp32 against 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from tests.parity import assert_close
from workloads import small_params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


LAYERS = [  # 16, 32 and 64 lanes a neighbour, scatter kernels (wide head; P > 7), both distances
    dict(T=3, C=8, H=10, W=11, HD=2, wt=2, ps=3, k=5), dict(T=2, C=16, H=8, W=9, ps=1, k=30, ws=7, dist_type=1),
    dict(T=2, C=40, H=7, W=9, HD=2, ps=2, k=7), dict(T=3, C=33, H=8, W=8, wt=2, ps=3, k=6, dist_type=1),
    dict(T=2, C=64, H=7, W=6, ps=1, k=9, stride0=2), dict(T=2, C=70, H=6, W=7, ps=1, k=5),
    dict(T=2, C=66, H=6, W=7, ps=3, k=4, dist_type=1), dict(T=2, C=4, H=9, W=9, ps=9, k=3),
    dict(T=2, C=8, H=6, W=7, HD=2, ps=1, k=1),  # a single neighbour: its weight is 1 whatever its score
]


def _rows(p, seed):
    """Scores and positions, a third of them bad in one of the ways, some rows wholly so; some scores not finite."""
    g = torch.Generator().manual_seed(seed)
    shp = B.out_shape(p)
    d = torch.randn(shp, generator=g)
    inds = torch.empty(shp + (3,))
    inds[..., 0] = torch.randint(0, p["T"], shp, generator=g).float()
    inds[..., 1:] = 2.5 * torch.randn(shp + (2,), generator=g)
    ways = [(0, -1.0), (0, float(p["T"])), (0, 0.5), (0, float("nan")), (0, float("-inf")), (1, 1e6), (1, float("nan")),
            (2, -1e6), (2, float("inf"))]
    pick = torch.randint(0, 3 * len(ways), shp, generator=g)
    pick[:, :, :, 0, :2] = torch.randint(0, len(ways), pick[:, :, :, 0, :2].shape, generator=g)
    for j, (col, val) in enumerate(ways):
        inds[..., col] = torch.where(pick == j, torch.full_like(d, val), inds[..., col])
    odd = torch.randint(0, 40, shp, generator=g)
    for j, val in enumerate((float("inf"), -float("inf"), float("nan"))):
        d = torch.where(odd == j, torch.full_like(d, val), d)
    return d, inds


@pytest.mark.parametrize("with_grad_dists", [False, True])
@pytest.mark.parametrize("kw", LAYERS, ids=range(len(LAYERS)))
def test_bad_positions(dev, kw, with_grad_dists):
    p = small_params(**kw)
    d, inds = _rows(p, 3)
    g = torch.Generator().manual_seed(4)
    q, k, v, go = (torch.randn(B.video_shape(p), generator=g) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), generator=g)
    gd = torch.randn(d.shape, generator=g) if with_grad_dists else None
    scale = 0.7
    to = lambda x: None if x is None else x.to(dev)  # noqa: E731
    print("positions", p, flush=True)
    args = [to(x) for x in (q, k, v, fl, d, inds, go)]
    gq, gk, gv, gf, gs = B.snls_backward_scores(*args, p, scale, grad_dists=to(gd))
    plain = B.snls_backward(*args, p, scale, grad_dists=to(gd))
    dl = d.double().requires_grad_()
    out = R.aggregate(v.double(), dl, inds, p, scale)
    assert_close(B.snls_aggregate(args[2], args[4], args[5], p, scale).cpu().numpy(), out.detach().numpy(), "out")
    want, = torch.autograd.grad((out * go.double()).sum(), dl)
    ok = R.bias_entries(inds, p, dict(radius=1, edges=[]))[-1] & d.isfinite()
    assert not bool(want[~d.isfinite()].any())
    bad = ~ok & d.isfinite()
    assert p["k"] == 1 or bool((want[bad].abs() > 1e-3).any())
    if with_grad_dists:  # counts where the neighbour is read, as for the gradients of q and k
        want = want + torch.where(ok, gd.double(), torch.zeros((), dtype=R.F64))
    assert_close(gs.cpu().numpy(), want.numpy(), "grad_scores")
    # the oracle knows bad frames; a bad displacement is the same to the library
    named = torch.where(ok[..., None], inds, torch.tensor([-1.0, 0.0, 0.0]))
    ref = oracle.backward(*(x.numpy() for x in (q, k, v, fl, d, named, go)), p, scale,
                          **({"grad_dists": gd.numpy()} if with_grad_dists else {}))
    for got, other, r, name in zip((gq, gk, gv, gf), plain, ref, ("grad_q", "grad_k", "grad_v", "grad_flows")):
        assert_close(got.cpu().numpy(), r, name)
        assert_close(other.cpu().numpy(), r, name)


def test_scores_gradient_is_the_difference(dev):
    """The gradient of bad neighbours' scores against differences of the library's own loss."""
    p = small_params(T=2, C=8, H=6, W=7, ps=3, k=4)
    d, inds = _rows(p, 8)
    g = torch.Generator().manual_seed(9)
    v, go = (torch.randn(B.video_shape(p), generator=g).to(dev) for _ in range(2))
    fl = torch.zeros(B.flow_shape(p), device=dev)
    dg, ig = d.to(dev), inds.to(dev)
    gs = B.snls_backward_scores(v, v, v, fl, dg, ig, go, p, 1.0)[4].cpu().double()
    ok = R.bias_entries(inds, p, dict(radius=1, edges=[]))[-1]
    bad = (~ok & d.isfinite()).nonzero()[::9][:12]
    assert len(bad) == 12
    h = 2.0 ** -4

    def loss(at, step):
        x = dg.clone()
        x[tuple(at)] += step
        return float((B.snls_aggregate(v, x, ig, p, 1.0).double() * go.double()).sum())

    for at in bad:
        # central difference: h^2 / 6 times a third derivative of at most 6 S (of a softmax weight), S the largest sum of
        # one query's terms, and fp32 outputs: 504 terms of rounding 2^-22 S over 2 h
        num = (loss(at, h) - loss(at, -h)) / (2 * h)
        S = float(gs.abs().max()) * 4
        assert abs(num - float(gs[tuple(at)])) <= S * (h * h + 504 * 2.0 ** -22 / (2 * h)), tuple(at)
