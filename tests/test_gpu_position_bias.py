"""The learned position bias and its training on the GPU against the plain
64-bit forms (tests/attention64.py).

Tolerances.  A biased score is one fp32 addition: equal to the fp32 sum bit by
bit.  A table entry sums n gradients in fp32, at most n - 1 roundings of
partial sums no larger than the sum of magnitudes: n * 2^-24 * sum |g|.  The
gradients of the whole layer have the parity bar of the library's backward
pass (tests/parity.py)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from tests.parity import assert_close
from workloads import small_params

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _neighbours(p, seed, odd=True):
    """Scores and positions with frames outside the clip and the window, odd frames, far and non-finite
    displacements, non-finite scores, displacements on the edges."""
    g = torch.Generator().manual_seed(seed)
    shp = B.out_shape(p)
    d = torch.randn(shp, generator=g)
    inds = torch.empty(shp + (3,))
    inds[..., 0] = torch.randint(-1, p["T"] + 1, shp, generator=g).float()
    inds[..., 1:] = 6 * torch.randn(shp + (2,), generator=g)
    edge = torch.tensor([0.0, -0.0, 0.5, -0.5, 2.0, -2.0, 7.5, -7.5, np.nextafter(np.float32(2.0), np.float32(0))])
    pick = torch.randint(0, 40, shp + (2,), generator=g)
    inds[..., 1:] = torch.where(pick < 9, edge[pick.clamp_max(8)], inds[..., 1:])
    if odd:
        flat_i, flat_d = inds.view(-1, 3), d.view(-1)
        n = flat_d.numel()
        for j, (col, val) in enumerate(((0, 0.5), (0, float("nan")), (0, 1e9), (0, float("-inf")), (1, 1e6), (2, -1e6),
                                        (1, float("nan")), (2, float("inf")), (1, 999999.0))):
            flat_i[(j * 7 + 3) % n, col] = val
        for j, val in enumerate((float("inf"), float("-inf"), float("nan"))):
            flat_d[(j * 11 + 1) % n] = val
    return d, inds


CASES = [  # (parameters, radius, edges)
    (dict(T=3, H=12, W=13, HD=2, k=4), 1, [0.5, 2.0, 7.5]),
    (dict(B=2, T=2, H=7, W=5, HD=4, C=8, k=3, stride0=2, dist_type=1), 2, [0.5, 1.0, 2.0, 4.0, 7.5]),
    (dict(T=1, H=1, W=1, k=1, ws=1, wt=0, ps=1), 0, []),
    (dict(T=4, H=9, W=11, k=0, ws=3, wt=1, ps=1), 0, [2.0]),  # every candidate kept
    (dict(T=2, H=33, W=65, k=9, ws=3, wt=1), 63, [0.5, 2.0]),
    (dict(B=1, T=5, H=64, W=70, HD=1, C=4, k=16, ws=5, wt=2), 2, [float(2 ** i) / 4 for i in range(13)]),  # 3645 buckets
    (dict(B=2, T=3, H=40, W=41, HD=2, k=30, ws=7, wt=1), 1, [0.5 + i for i in range(16)]),  # 3267 buckets
    (dict(T=2, H=30, W=31, HD=3, C=9, k=5, dist_type=1), 1, [0.5, 2.0, 7.5, 8.0]),
]


@pytest.mark.parametrize("kw,radius,edges", CASES, ids=range(len(CASES)))
def test_bias_and_table_gradient(dev, kw, radius, edges):
    p, bias = small_params(**kw), dict(radius=radius, edges=edges)
    d, inds = _neighbours(p, 5)
    g = torch.Generator().manual_seed(6)
    table = torch.randn(B.bias_table_shape(bias, p["HD"]), generator=g)
    grad = torch.randn(d.shape, generator=g)
    dg, ig, tg, gg = (x.to(dev) for x in (d, inds, table, grad))
    print("bias", p, bias["radius"], len(edges), flush=True)
    out = B.snls_bias(dg, ig, tg, p, bias)
    assert torch.equal(out.cpu().view(torch.int32), R.biased(d, inds, table, p, bias).view(torch.int32))
    same = dg.clone()
    B.snls_bias(same, ig, tg, p, bias, out=same)
    assert torch.equal(same.view(torch.int32), out.view(torch.int32))
    got = B.snls_bias_backward(gg, dg, ig, p, bias)
    again = B.snls_bias_backward(gg, out, ig, p, bias)  # the biased scores are finite at the same neighbours
    assert torch.equal(got, again)
    ref, cnt, mag = R.table_grad(grad, d, inds, p, bias, p["HD"])
    assert bool(((got.cpu().double() - ref).abs() <= cnt * EPS * mag + 1e-300).all())


def test_table_entries_not_finite(dev):
    """A table entry of -inf takes its bucket out of the softmax, the lowest value keeps it; the score of an invalid
    candidate stays as it is whatever the table holds; NaN and infinite gradients of neighbours that do not count
    stay out of the sums."""
    p, bias = small_params(T=3, H=8, W=9, k=4), dict(radius=1, edges=[0.5, 2.0])
    d, inds = _neighbours(p, 9)
    table = torch.randn(B.bias_table_shape(bias, 1))
    table[0, 1, 2, 2], table[0, 0, 1, 1], table[0, 2, 3, 3] = -float("inf"), torch.finfo(torch.float32).min, float("inf")
    out = B.snls_bias(d.to(dev), inds.to(dev), table.to(dev), p, bias).cpu()
    want = R.biased(d, inds, table, p, bias)
    assert torch.equal(out.view(torch.int32), want.view(torch.int32))
    grad = torch.randn(d.shape)
    ref, cnt, mag = R.table_grad(grad, d, inds, p, bias, 1)
    ok = R.bias_entries(inds, p, bias)[-1] & d.isfinite()
    grad = torch.where(ok, grad, torch.full_like(grad, float("nan")))
    got = B.snls_bias_backward(grad.to(dev), d.to(dev), inds.to(dev), p, bias).cpu()
    assert bool(((got.double() - ref).abs() <= cnt * EPS * mag + 1e-300).all())


def test_many_into_one_bucket(dev):
    """Two million gradients of one bucket, all of one sign: the partial sums stay short."""
    p, bias = small_params(T=2, C=4, H=160, W=160, k=40, ws=7, wt=1, ps=1), dict(radius=0, edges=[])
    shp = B.out_shape(p)
    inds = torch.zeros(shp + (3,), device=dev)
    grad = torch.rand(shp, device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    got = float(B.snls_bias_backward(grad, torch.zeros(shp, device=dev), inds, p, bias))
    want = float(grad.double().sum())
    # a lane's copy of an entry sums at most a slice's share; 1280 slices are added in 64 bits
    assert abs(got - want) <= 2e-5 * want


LAYERS = [  # binned backward pass, its atomic form (wide head), squared L2, heads, strides, single pixels
    dict(T=3, C=8, H=10, W=11, HD=2, ws=3, wt=1, ps=3, k=4),
    dict(T=2, C=70, H=7, W=8, ws=3, wt=1, ps=1, k=5),
    dict(T=3, C=6, H=9, W=10, ws=5, wt=1, ps=2, k=6, dist_type=1, stride0=2),
    dict(T=2, C=70, H=6, W=7, ws=3, wt=1, ps=3, k=3, dist_type=1),
    dict(B=2, T=3, C=16, H=9, W=7, HD=4, ws=5, wt=2, ps=1, k=20),
    # the channels at which a neighbour's lanes change, numbers of neighbours that fill no group of lanes
    dict(T=2, C=16, H=9, W=8, ws=5, wt=1, ps=3, k=7), dict(T=2, C=17, H=8, W=9, ws=5, wt=1, ps=2, k=5, dist_type=1),
    dict(T=2, C=64, H=7, W=9, HD=2, ws=5, wt=1, ps=1, k=9, stride0=2),
    dict(T=2, C=32, H=8, W=8, ws=3, wt=1, ps=7, k=3, dist_type=1), dict(T=2, C=33, H=8, W=8, ws=5, wt=1, ps=3, k=6),
    dict(T=2, C=32, H=9, W=12, HD=2, ws=3, wt=1, ps=5, k=1),
]


@pytest.mark.parametrize("with_grad_dists", [False, True])
@pytest.mark.parametrize("kw", LAYERS, ids=range(len(LAYERS)))
def test_training_step(dev, kw, with_grad_dists):
    """Search, bias, aggregation and their gradients, as a layer runs them: against the oracle (q, k, v, flows) and
    64-bit automatic differentiation of the aggregation (scores, table)."""
    p = small_params(**kw)
    bias = dict(radius=p["wt"], edges=[0.5, 1.5, 4.0])
    r = np.random.default_rng(3)
    vid = (p["B"], p["T"], p["C"], p["H"], p["W"])
    q, k, v, go = (r.standard_normal(vid, dtype=np.float32) for _ in range(4))
    fl = r.uniform(-3, 3, (p["B"], p["T"], 2 * p["wt"], 2, p["H"], p["W"])).astype(np.float32)
    table = r.standard_normal(B.bias_table_shape(bias, p["HD"])).astype(np.float32)
    scale = 0.2
    to = lambda a: torch.from_numpy(a).to(dev)  # noqa: E731
    qg, kg, vg, fg, gg, tg = map(to, (q, k, v, fl, go, table))
    print("train", p, flush=True)
    d, i = B.snls_search(qg, kg, fg, p)
    db = B.snls_bias(d, i, tg, p, bias)
    gd = torch.randn(d.shape, generator=torch.Generator().manual_seed(4)) if with_grad_dists else None
    out = B.snls_aggregate(vg, db, i, p, scale)
    gq, gk, gv, gf, gs = B.snls_backward_scores(qg, kg, vg, fg, db, i, gg, p, scale,
                                                grad_dists=gd.to(dev) if with_grad_dists else None)
    gt = B.snls_bias_backward(gs, db, i, p, bias)
    dbc, ic = db.cpu(), i.cpu()
    dl = dbc.double().requires_grad_()
    o64 = R.aggregate(torch.from_numpy(v).double(), dl, ic, p, scale)
    assert_close(out.cpu().numpy(), o64.detach().numpy(), "out")
    ds, = torch.autograd.grad((o64 * torch.from_numpy(go).double()).sum(), dl)
    if with_grad_dists:
        ok = R.bias_entries(ic, p, bias)[-1] & dbc.isfinite()
        ds = ds + torch.where(ok, gd.double(), torch.zeros((), dtype=R.F64))
    assert_close(gs.cpu().numpy(), ds.numpy(), "grad_scores")
    want = oracle.backward(q, k, v, fl, dbc.numpy(), ic.numpy(), go, p, scale,
                           **({"grad_dists": gd.numpy()} if with_grad_dists else {}))
    for got, ref, name in zip((gq, gk, gv, gf), want, ("grad_q", "grad_k", "grad_v", "grad_flows")):
        assert_close(got.cpu().numpy(), ref, name)
    # the table's gradient: exact sums of the library's own score gradients, and the layer's to the parity bar
    ref, cnt, mag = R.table_grad(gs.cpu(), dbc, ic, p, bias, p["HD"])
    assert bool(((gt.cpu().double() - ref).abs() <= cnt * EPS * mag + 1e-300).all())
    full, _, fmag = R.table_grad(ds, dbc, ic, p, bias, p["HD"])
    rms = float(ds.square().mean().sqrt())
    assert bool(((gt.cpu().double() - full).abs() <= 1e-4 * (fmag + cnt * rms)).all())


def test_scores_do_not_change_the_other_gradients(dev):
    """snls_backward_scores gives snls_backward's gradients; one neighbour's dV is free of atomics: bit-identical."""
    p = small_params(T=3, C=16, H=20, W=21, ws=5, wt=1, ps=3, k=6)
    g = torch.Generator(device=dev).manual_seed(2)
    q, k, v, go = (torch.randn(B.video_shape(p), device=dev, generator=g) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), device=dev, generator=g)
    d, i = B.snls_search(q, k, fl, p)
    a = B.snls_backward(q, k, v, fl, d, i, go, p, 0.1)
    b = B.snls_backward_scores(q, k, v, fl, d, i, go, p, 0.1)
    for x, y in zip(a, b):
        assert_close(y.cpu().numpy(), x.cpu().numpy(), "gradient", rel=1e-5)


def test_streams_and_graph(dev):
    """The three calls on a side stream and in a graph that is replayed with new inputs."""
    p, bias = small_params(T=3, C=8, H=20, W=22, HD=2, k=5), dict(radius=1, edges=[0.5, 2.0])
    d, inds = _neighbours(p, 1)
    dg, ig = d.to(dev), inds.to(dev)
    gen = torch.Generator(device=dev).manual_seed(8)
    table = torch.randn(B.bias_table_shape(bias, 2), device=dev, generator=gen)
    grad = torch.randn(d.shape, device=dev, generator=gen)
    out, gt = torch.empty_like(dg), torch.empty_like(table)
    ws = B.workspace_for(B.SNLS_OP_BIAS_BACKWARD, p, dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.snls_bias(dg, ig, table, p, bias, out=out)
        B.snls_bias_backward(grad, dg, ig, p, bias, grad_table=gt, workspace=ws)
    side.synchronize()
    assert torch.equal(out.view(torch.int32), B.snls_bias(dg, ig, table, p, bias).view(torch.int32))
    assert torch.equal(gt, B.snls_bias_backward(grad, dg, ig, p, bias))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.snls_bias(dg, ig, table, p, bias, out=out)
        B.snls_bias_backward(grad, dg, ig, p, bias, grad_table=gt, workspace=ws)
    for _ in range(3):
        table.normal_(generator=gen)
        grad.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int32), B.snls_bias(dg, ig, table, p, bias).view(torch.int32))
        assert torch.equal(gt, B.snls_bias_backward(grad, dg, ig, p, bias))


@pytest.mark.parametrize("HD", [4095, 4097, 9000])
def test_many_heads(dev, HD):
    """More heads than waves on the chip: one slice a head."""
    p, bias = small_params(T=2, C=HD, H=3, W=3, HD=HD, k=3), dict(radius=0, edges=[1.0])
    d, inds = _neighbours(p, 3)
    g = torch.Generator().manual_seed(4)
    table = torch.randn(B.bias_table_shape(bias, HD), generator=g)
    grad = torch.randn(d.shape, generator=g)
    out = B.snls_bias(d.to(dev), inds.to(dev), table.to(dev), p, bias)
    assert torch.equal(out.cpu().view(torch.int32), R.biased(d, inds, table, p, bias).view(torch.int32))
    got = B.snls_bias_backward(grad.to(dev), d.to(dev), inds.to(dev), p, bias).cpu()
    ref, cnt, mag = R.table_grad(grad, d, inds, p, bias, HD)
    assert bool(((got.double() - ref).abs() <= cnt * EPS * mag + 1e-300).all())


def test_training_step_in_a_graph(dev):
    """Search to table gradient in one graph on one workspace each, replayed with new inputs against the eager step."""
    p = small_params(T=3, C=16, H=12, W=13, HD=2, ws=5, wt=1, ps=3, k=6)
    bias = dict(radius=1, edges=[0.5, 2.0])
    gen = torch.Generator(device=dev).manual_seed(12)
    q, k, v, go = (torch.randn(B.video_shape(p), device=dev, generator=gen) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), device=dev, generator=gen)
    table = torch.randn(B.bias_table_shape(bias, 2), device=dev, generator=gen)

    def step():
        d, i = B.snls_search(q, k, fl, p)
        d = B.snls_bias(d, i, table, p, bias, out=d)
        out = B.snls_aggregate(v, d, i, p, 0.2)
        grads = B.snls_backward_scores(q, k, v, fl, d, i, go, p, 0.2)
        return (out,) + grads + (B.snls_bias_backward(grads[4], d, i, p, bias),)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        for t in (q, k, v, go, fl, table):
            t.normal_(generator=gen)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for a, b, name in zip(held, want, ("out", "grad_q", "grad_k", "grad_v", "grad_flows", "grad_scores",
                                           "grad_table")):
            assert_close(a.cpu().numpy(), b.cpu().numpy(), name, rel=1e-5)
