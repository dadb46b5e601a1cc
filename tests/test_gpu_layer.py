"""Norm, dropout, rotary positions and 8-bit projections against their plain
64-bit forms, element by element within bounds derived there."""
import math

import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import layer64 as R
from workloads import small_params

pytestmark = pytest.mark.gpu
U = R.U


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _feat(g, shape, spread=1.0, offset=0.5):
    x = torch.randn(shape, generator=g)
    c = shape[-3] if len(shape) > 2 else shape[1]
    at = [1] * len(shape)
    at[-3 if len(shape) > 2 else 1] = c
    return x * torch.exp(spread * torch.randn(at, generator=g)) + offset * torch.randn(at, generator=g)


def _within(got, want, bound, what):
    off = (got.detach().cpu().double() - want).abs()
    over = off > bound
    assert not bool(over.any()) and not bool(off.isnan().any()), "%s: %d of %d out of bounds, worst %.3g over %.3g" % (
        what, int(over.sum()), over.numel(), float(off[over].max()), float(bound.expand_as(off)[over].min()))


def _to(dev, *ts):
    return [None if t is None else t.to(dev) for t in ts]


RNG = (-0x1234567890abcde, 77)

# frames or tokens: odd pixel counts, channel counts around the lanes and past what registers hold
SHAPES = [(1, 1, 1, 1, 1), (1, 1, 3, 1, 1), (1, 1, 16, 1, 2), (2, 3, 16, 13, 17), (1, 2, 48, 9, 7), (1, 1, 64, 16, 16),
          (1, 1, 64, 5, 103), (2, 1, 65, 8, 33), (1, 1, 192, 15, 17), (1, 2, 256, 6, 43), (1, 1, 257, 3, 22),
          (1, 1, 300, 9, 32), (1, 1, 1030, 3, 23), (3, 20, 1, 1), (2, 100, 1, 3),
          (1, 1), (1, 7), (1, 64), (2, 192), (3, 193), (65, 48), (257, 64), (300, 16), (5, 256), (7, 1000), (3, 1024),
          (2, 1500), (1000, 20), (1, 2, 128, 9, 15), (1, 1, 129, 8, 12), (2, 1, 384, 5, 13), (1, 1, 385, 4, 16), (1, 1, 512, 3, 20),
          (1, 1, 513, 2, 9), (4, 2050)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("how", ["plain", "bare", "sum", "drop"])
def test_norm(dev, shape, how):
    g = _gen(sum(shape))
    x, br = _feat(g, shape), torch.randn(shape, generator=g)
    C = shape[1] if len(shape) == 2 else shape[-3]
    gamma, beta = (None, None) if how == "bare" else (torch.randn(C, generator=g), torch.randn(C, generator=g))
    drop = 0.3 if how == "drop" else 0.0
    branch = br if how in ("sum", "drop") else None
    eps = 1e-5
    rng = torch.tensor(RNG, dtype=torch.int64)
    y, total, stats = B.snls_norm(*_to(dev, x, gamma, beta), eps=eps, branch=_to(dev, branch)[0], drop=drop,
                                  rng=rng.to(dev), site=9)
    if branch is None:
        want, err = x.double(), torch.zeros_like(x, dtype=torch.float64)
        assert total.data_ptr() != y.data_ptr() and torch.equal(total.cpu(), x)
    else:
        add = R.dropout(branch, RNG, drop, 9)
        want = x.double() + add
        err = 2 * U * add.abs() + U * want.abs()  # the factor, the product, the sum
        _within(total, want, err, "total")
    wy, wm, wr = R.norm(want, gamma, beta, eps)
    by, bm, brs = R.norm_bound(want, gamma, beta, eps, err)
    _within(y, wy, by, "y")
    _within(stats[0], wm, bm, "mean")
    _within(stats[1], wr, brs, "rstd")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("how", ["plain", "bare", "sum", "drop"])
def test_norm_backward(dev, shape, how):
    g = _gen(sum(shape) + 1)
    total, gy, gt = _feat(g, shape), torch.randn(shape, generator=g), torch.randn(shape, generator=g)
    C = shape[1] if len(shape) == 2 else shape[-3]
    gamma = None if how == "bare" else torch.randn(C, generator=g)
    drop = 0.3 if how == "drop" else 0.0
    gtotal = gt if how in ("sum", "drop") else None
    _, mean, rstd = R.norm(total.double(), None, None, 1e-5)
    stats = torch.stack([mean, rstd]).float()
    rng = torch.tensor(RNG, dtype=torch.int64).to(dev)
    args = _to(dev, gy, total, stats, gamma)
    gx, gb, gg, gbt = B.snls_norm_backward(*args, grad_total=_to(dev, gtotal)[0], drop=drop, rng=rng, site=4)
    (wx, wg, wb), (ex, eg, eb) = R.norm_backward(gy, total, stats, gamma, gtotal)
    _within(gx, wx, ex, "grad_x")
    _within(gg, wg, eg, "grad_gamma")
    _within(gbt, wb, eb, "grad_beta")
    if drop == 0:
        assert gb.data_ptr() == gx.data_ptr()
        again = B.snls_norm_backward(*args, grad_total=_to(dev, gtotal)[0], grad_branch=torch.empty_like(gx), weights=False)
        assert torch.equal(again[0], gx) and torch.equal(again[1], gx) and again[2] is None and again[3] is None
    else:
        keep = R.keep_mask(shape, RNG, drop, 4)
        assert bool((gb.cpu()[~keep] == 0).all())
        f = 1 / (1 - R.drop32(drop))
        _within(gb, torch.where(keep, wx * f, 0.0), torch.where(keep, (ex + 2 * U * wx.abs()) * f * (1 + 4 * U), 0.0), "grad_branch")


def test_norm_in_place(dev):
    g = _gen(8)
    for shape in ((1, 2, 48, 9, 7), (2, 1, 300, 5, 9), (33, 64), (3, 1500)):
        x, br, gy, gt = (torch.randn(shape, generator=g).to(dev) for _ in range(4))
        rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
        y, total, stats = B.snls_norm(x, branch=br, drop=0.25, rng=rng)
        for target in (0, 1):
            a, b = x.clone(), br.clone()
            t = (a, b)[target]
            y2, t2, st2 = B.snls_norm(a, branch=b, drop=0.25, rng=rng, total=t)
            assert t2 is t and torch.equal(t, total) and torch.equal(y2, y) and torch.equal(st2, stats)
        y1 = B.snls_norm(x)[0]
        a = x.clone()
        assert torch.equal(B.snls_norm(a, y=a)[0], y1)
        want = B.snls_norm_backward(gy, total, stats, grad_total=gt, drop=0.25, rng=rng)
        for target in (0, 1):
            a, b = gy.clone(), gt.clone()
            got = B.snls_norm_backward(a, total, stats, grad_total=b, drop=0.25, rng=rng, grad_x=(a, b)[target])
            assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_norm_special_values(dev):
    x = torch.randn(1, 1, 24, 5, 13, generator=_gen(2))
    x[0, 0, 3, 1, 2] = float("nan")
    x[0, 0, 5, 4, 0] = float("inf")
    x[0, 0, :, 2, 2] = 7.0  # a pixel without variance
    y, _, stats = B.snls_norm(x.to(dev), eps=1e-5)
    bad = torch.zeros(5, 13, dtype=torch.bool)
    bad[1, 2] = bad[4, 0] = True
    assert bool(y.cpu()[0, 0, :, bad].isnan().any(0).all()) and not bool(y.cpu()[0, 0, :, ~bad].isnan().any())
    assert float(y[0, 0, :, 2, 2].abs().max()) <= 24 * U * 7 * (1 / math.sqrt(1e-5)) and float(stats[0, 0, 0, 2, 2]) == 7.0
    # far from zero, little variance: differences from the mean are squared
    z = torch.randn(1, 1, 64, 4, 16, generator=_gen(3)) * 0.01 + 1000
    y, _, _ = B.snls_norm(z.to(dev), eps=0.0)
    wy, _, _ = R.norm(z.double(), None, None, 0.0)
    _within(y, wy, R.norm_bound(z.double(), None, None, 0.0, torch.zeros_like(z, dtype=torch.float64))[0], "offset")
    assert float((y.cpu().double() - wy).abs().max()) < 0.1


def test_dropped_nan_does_not_show(dev):
    shape = (1, 1, 16, 6, 11)
    keep = R.keep_mask(shape, RNG, 0.5, 2)
    br = torch.ones(shape)
    br[~keep] = float("nan")
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    x = torch.randn(shape, generator=_gen(1)).to(dev)
    out = B.snls_dropout(br.to(dev), rng, 0.5, site=2)
    assert torch.equal(out.cpu(), torch.where(keep, 2.0, 0.0))
    y, total, _ = B.snls_norm(x, branch=br.to(dev), drop=0.5, rng=rng, site=2)
    assert not bool(total.isnan().any()) and not bool(y.isnan().any())


@pytest.mark.parametrize("n", [1, 2, 3, 5, 255, 1023, 4099, 100003])
@pytest.mark.parametrize("drop", [0.0, 0.1, 0.5, 0.999, 1e-10])
def test_dropout(dev, n, drop):
    g = _gen(n)
    x, res = torch.randn(n, generator=g), torch.randn(n, generator=g)
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    out = B.snls_dropout(x.to(dev), rng, drop, site=0xffffffff)
    want = R.dropout(x, RNG, drop, 0xffffffff)
    assert torch.equal(out.cpu() == 0, want == 0)
    _within(out, want, 2 * U * want.abs(), "dropout")
    both = B.snls_dropout(x.to(dev), rng, drop, site=0xffffffff, residual=res.to(dev))
    s = want + res.double()
    _within(both, s, 2 * U * want.abs() + U * s.abs(), "residual")
    a, b = x.to(dev), res.to(dev)
    assert torch.equal(B.snls_dropout(a, rng, drop, site=0xffffffff, residual=b, out=b), both)
    assert torch.equal(B.snls_dropout(a, rng, drop, site=0xffffffff, out=a), out)


def test_dropout_masks_differ_by_seed_step_and_site_and_agree_with_the_norm(dev):
    shape = (2, 2, 19, 7, 9)
    one = torch.ones(shape, device=dev)

    def mask(seed, step, site):
        return B.snls_dropout(one, torch.tensor([seed, step], dtype=torch.int64, device=dev), 0.5, site=site) > 0

    base = mask(5, 6, 7)
    for other in ((5 + 2 ** 32, 6, 7), (6, 6, 7), (5, 7, 7), (5, 6, 8)):
        share = float((mask(*other) == base).double().mean())
        assert abs(share - 0.5) < 6 * 0.5 / math.sqrt(base.numel())  # six standard deviations
    assert torch.equal(mask(5, 6 + 2 ** 32, 7), base)
    rng = torch.tensor([5, 6], dtype=torch.int64, device=dev)
    _, total, _ = B.snls_norm(torch.zeros(shape, device=dev), branch=one, drop=0.5, rng=rng, site=7)
    assert torch.equal(total > 0, base)
    rows = one.reshape(-1, 19 * 9)
    _, total, _ = B.snls_norm(torch.zeros_like(rows), branch=rows, drop=0.5, rng=rng, site=7)
    assert torch.equal((total > 0).reshape(shape), base)


def test_dropout_past_32_bits(dev):
    """Element 2^34 and beyond: the counter's second word."""
    n = (1 << 34) + 21
    if torch.cuda.mem_get_info()[0] < 5 * n:
        pytest.skip("not enough memory")
    x = torch.ones(n, device=dev)
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    B.snls_dropout(x, rng, 0.5, site=1, out=x)
    for first in (0, (1 << 32) - 8, (1 << 34) - 13):
        m = min(4096, n - first)
        want = torch.from_numpy(R.words(first, m, RNG[0], RNG[1], 1) >= 2 ** 31)
        assert torch.equal(x[first:first + m].cpu() > 0, want)
    del x
    torch.cuda.empty_cache()


ROTS = [
    dict(B=1, T=1, C=2, H=1, W=1, HD=1, pairs=(1, 0, 0)),
    dict(B=1, T=2, C=8, H=3, W=5, HD=1, pairs=(0, 2, 2)),
    dict(B=2, T=3, C=48, H=13, W=17, HD=2, pairs=(3, 4, 5)),
    dict(B=1, T=2, C=40, H=9, W=66, HD=2, pairs=(2, 3, 2)),  # channels left over, an even and an odd number
    dict(B=1, T=1, C=57, H=7, W=64, HD=3, pairs=(1, 4, 4)),
    dict(B=1, T=2, C=64, H=33, W=103, HD=1, pairs=(8, 12, 12)),
    dict(B=1, T=1, C=256, H=4, W=9, HD=1, pairs=(0, 0, 128)),
    dict(B=1, T=1, C=24, H=5, W=2100, HD=1, pairs=(2, 3, 3)),
    dict(B=1, T=1, C=24, H=700, W=3, HD=1, pairs=(2, 3, 3)),
    dict(B=1, T=1, C=12, H=6, W=7, HD=2, pairs=(0, 0, 0)),
]


@pytest.mark.parametrize("rp", ROTS, ids=range(len(ROTS)))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("far", [False, True])
def test_rotate(dev, rp, interleaved, far):
    rp = dict(rp, theta=(10000.0, 100.0, 30.0), interleaved=interleaved)
    if far:
        rp.update(row0=-5000, col0=123456)
    g = _gen(rp["C"])
    shp = B.video_shape(rp)
    q, k = torch.randn(shp, generator=g), torch.randn(shp, generator=g)
    times = torch.randint(-2 ** 24, 2 ** 24, (rp["B"], rp["T"]), generator=g) if far else None
    inverse = far
    qo, ko = B.snls_rotate(*_to(dev, q, k), rp, times=_to(dev, times)[0], inverse=inverse)
    most = 2.0 ** 24 if far else 2200.0
    for got, x in ((qo, q), (ko, k)):
        _within(got, R.rotate_video(x, times, rp, inverse), R.rotate_bound(x, rp, shp, most), "rotate")
    a, b = _to(dev, q, k)
    td = _to(dev, times)[0]
    a2, b2 = B.snls_rotate(a, b, rp, times=td, inverse=inverse, q_out=a, k_out=b)
    assert a2 is a and torch.equal(a, qo) and torch.equal(b, ko)
    alone, none = B.snls_rotate(q.to(dev), None, rp, times=td, inverse=inverse)
    assert none is None and torch.equal(alone, qo)


@pytest.mark.parametrize("n", [1, 2, 63, 500])
@pytest.mark.parametrize("rp", [ROTS[2], ROTS[3], ROTS[4], ROTS[6], ROTS[9]], ids=[2, 3, 4, 6, 9])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_points(dev, n, rp, interleaved):
    rp = dict(rp, theta=(10000.0, 100.0, 30.0), interleaved=interleaved, row0=3, col0=-2)
    g = _gen(n + rp["C"])
    q = torch.randn(n, rp["C"], generator=g)
    pts = torch.stack([torch.randint(-1, rp[m] + 1, (n,), generator=g) for m in ("B", "H", "W")], 1).to(torch.int32)
    times = torch.randint(-10000, 10 ** 6, (rp["B"],), generator=g)
    for t in (times, None):
        for inverse in (False, True):
            out = B.snls_rotate_points(*_to(dev, q, pts), rp, times=_to(dev, t)[0], inverse=inverse)
            want = R.rotate_points(q, pts, t, rp, inverse)
            _within(out, want, R.rotate_bound(q, rp, q.shape, 1e6), "points")
            assert bool((out.cpu()[(want == 0).all(1)] == 0).all())
            a = q.to(dev)
            assert torch.equal(B.snls_rotate_points(a, pts.to(dev), rp, times=_to(dev, t)[0], inverse=inverse, out=a), out)


# (shape of x, cout, parts): channels around the matrix instructions' steps, odd pixels
PROJ = [((1, 1, 1, 1, 1), 1, 1), ((1, 2, 16, 5, 7), 48, 3), ((2, 1, 64, 9, 33), 192, 3), ((1, 1, 48, 11, 12), 33, 1),
        ((1, 1, 33, 3, 41), 66, 2), ((1, 1, 192, 8, 9), 64, 1), ((1, 1, 250, 4, 8), 100, 4), ((1, 1, 256, 8, 8), 256, 2),
        ((1, 1, 300, 5, 5), 31, 1), ((1, 1, 1024, 3, 11), 40, 2), ((2, 3, 100, 1, 3), 70, 2), ((1, 1, 16, 5, 8), 2100, 3), ((1, 2, 384, 4, 32), 390, 2), ((1, 1, 20, 1, 64), 2048, 1),
        ((1, 3, 240, 8, 16), 96, 3), ((1, 2, 1024, 8, 8), 200, 2), ((2, 1, 992, 5, 7), 65, 1), ((100, 384), 384, 2),
        ((33, 512), 129, 1), ((70, 1024), 64, 1), ((65, 208), 36, 3), ((1, 1, 1001, 3, 47), 300, 2), ((40, 1001), 300, 1), ((1, 2, 250, 4, 37), 700, 1),
        ((1, 1), 1, 1), ((1, 192), 576, 3), ((2, 64), 192, 3), ((33, 48), 144, 3), ((65, 20), 34, 2), ((1, 1023), 96, 1),
        ((130, 256), 300, 3), ((1, 1024), 4097, 1), ((1000, 16), 32, 1), ((3, 130), 5, 5)]


@pytest.mark.parametrize("case", PROJ, ids=str)
def test_project(dev, case):
    shape, cout, parts = case
    g = _gen(cout)
    x = _feat(g, shape)
    cin = shape[1] if len(shape) == 2 else shape[-3]
    w = torch.randn(cout, cin, generator=g)
    codes, scales = B.snls_project_pack(w.to(dev))
    wc, ws = R.quantise(w)
    assert torch.equal(codes.cpu().double(), wc) and torch.equal(scales.cpu().double(), ws)
    for bias in (None, torch.randn(cout, generator=g)):
        out = B.snls_project(x.to(dev), codes, scales, bias=_to(dev, bias)[0], parts=parts)
        want, err = R.project(x, codes.cpu(), scales.cpu(), bias, parts)
        assert out.shape == want.shape
        _within(out, want, err, "project")


# outputs that no cache holds, of planes that share cache lines: (shape of x, cout, parts, floats before the output)
BIG = [((1, 1, 32, 470, 855), 200, 1, 0), ((1, 3, 64, 271, 483), 192, 3, 0), ((2, 1, 192, 152, 153), 1536, 2, 1),
       ((1, 1, 16, 740, 740), 128, 1, 5), ((1, 1, 96, 480, 512), 288, 3, 3), ((8000, 64, 3, 11), 256, 2, 0),
       ((4400, 128, 1, 31), 512, 4, 31), ((1, 1, 48, 480, 512), 300, 1, 32)]


@pytest.mark.parametrize("case", BIG, ids=str)
def test_project_past_the_caches(dev, case):
    """The same values as the pixels give as a list of tokens, and nothing beside them."""
    shape, cout, parts, before = case
    cin = shape[-3]
    g = torch.Generator(device=dev).manual_seed(cout)
    x = torch.randn(shape, generator=g, device=dev)
    x.view(-1, cin, shape[-2] * shape[-1])[0, 3, 17] = float("nan")
    codes, scales = B.snls_project_pack(torch.randn(cout, cin, generator=g, device=dev))
    bias = torch.randn(cout, generator=g, device=dev)
    n = cout * (x.numel() // cin)
    room = torch.full((n + before + 64,), -7.5, device=dev)
    out = room[before:before + n].view((parts,) + shape[:-3] + (cout // parts,) + shape[-2:])
    B.snls_project(x, codes, scales, bias=bias, parts=parts, out=out)
    tokens = x.view(-1, cin, shape[-2] * shape[-1]).transpose(1, 2).reshape(-1, cin).contiguous()
    want = B.snls_project(tokens, codes, scales, bias=bias, parts=parts)
    want = want.view(parts, -1, shape[-2] * shape[-1], cout // parts).transpose(2, 3)
    got = out.view(want.shape)
    assert bool(((got == want) | (got.isnan() & want.isnan())).all()) and int(got.isnan().sum()) == cout
    assert bool((room[:before] == -7.5).all()) and bool((room[before + n:] == -7.5).all())


def test_project_special_tokens(dev):
    """Halves next to their ties, tokens of zeros, of tiny and large values, infinities and NaN."""
    g = _gen(4)
    x = torch.randn(70, 40, generator=g)
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 7] = float("-inf")
    x[3] *= 1e-38
    x[4] *= 1e33
    x[5] = 1e-45
    for t in range(8, 70):  # codes at halves, a step of fp32 to either side
        s = torch.tensor(float(2.0 ** (t % 9 - 4)) * (1 + t / 97), dtype=torch.float32)
        h = (torch.randint(-126, 126, (40,), generator=g).float() + 0.5) * s
        x[t] = torch.where(torch.rand(40, generator=g) < 0.5, torch.nextafter(h, torch.zeros_like(h)), h)
        x[t, t % 40] = 127 * s
    w = torch.randn(24, 40, generator=g)
    w[3] = 0
    w[5, 2] = float("nan")
    codes, scales = B.snls_project_pack(w.to(dev))
    wc, ws = R.quantise(w)
    assert torch.equal(codes.cpu().double(), wc) and torch.equal(scales.cpu().double().isnan(), ws.isnan())
    eye = torch.eye(40, dtype=torch.int8, device=dev)  # the codes themselves
    out = B.snls_project(x.to(dev), eye, torch.ones(40, device=dev)).cpu()[0].double()
    qc, qs = R.quantise(x)
    ok = qs.isfinite()
    assert bool(out[~ok].isnan().all()) and ok.sum() == 68
    assert torch.equal(torch.round(out[ok] / qs[ok][:, None]), qc[ok])
    frames = x.t().reshape(1, 40, 70, 1).contiguous()
    same = B.snls_project(frames.to(dev), eye, torch.ones(40, device=dev)).cpu()[0, 0, :, :, 0].t().double()
    assert torch.equal(same[ok], out[ok]) and bool(same[~ok].isnan().all())


def test_empty_lists(dev):
    x = torch.empty(0, 8, device=dev)
    y, total, stats = B.snls_norm(x)
    assert y.shape == (0, 8) and stats.shape == (2, 0)
    gx, gb, gg, gbt = B.snls_norm_backward(x, x, stats)
    assert gx.shape == (0, 8) and float(gg.abs().max()) == 0 and float(gbt.abs().max()) == 0
    assert B.snls_dropout(x, None, 0.0).shape == (0, 8)
    rp = dict(B=1, T=1, C=8, H=2, W=2, HD=1, pairs=(1, 1, 1), theta=(10.0, 10.0, 10.0))
    assert B.snls_rotate_points(x, torch.empty(0, 3, dtype=torch.int32, device=dev), rp).shape == (0, 8)
    codes, scales = B.snls_project_pack(torch.randn(6, 8, device=dev))
    assert B.snls_project(x, codes, scales, parts=2).shape == (2, 0, 3)


def test_results_do_not_depend_on_scheduling(dev):
    g = torch.Generator(device=dev).manual_seed(6)
    x, gy = (torch.randn(2, 3, 48, 67, 91, generator=g, device=dev) for _ in range(2))
    _, _, stats = B.snls_norm(x)
    want = B.snls_norm_backward(gy, x, stats)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(B.snls_norm_backward(gy, x, stats), want))


def test_tensors_past_32_bits(dev):
    """4.4 thousand million elements: the far end of every call."""
    B_, C, H, W = 2, 68, 5700, 5700
    if torch.cuda.mem_get_info()[0] < 130e9:
        pytest.skip("not enough memory")
    shp = (B_, 1, C, H, W)
    g = torch.Generator(device=dev).manual_seed(2)
    x, br = (torch.randn(shp, generator=g, device=dev) for _ in range(2))
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    end = (B_ - 1, 0, slice(None), H - 1, slice(W - 300, W))
    first = ((B_ - 1) * C * H + H - 1) * W + W - 300
    keep = torch.stack([torch.from_numpy(R.words(first + c * H * W, 300, RNG[0], RNG[1], 3) >= 2 ** 30) for c in range(C)])
    cut = lambda t: t[end].cpu().double()[:, None, :]  # (C, 1, 300)  # noqa: E731
    y, total, st = B.snls_norm(x, branch=br, drop=0.25, rng=rng, site=3)
    add = torch.where(keep[:, None], cut(br) / 0.75, 0.0)
    want = cut(x) + add
    err = 2 * U * add.abs() + U * want.abs()
    _within(total[end][:, None], want, err, "total")
    _within(y[end][:, None], R.norm(want, None, None, 1e-5)[0], R.norm_bound(want, None, None, 1e-5, err)[0], "y")
    gx, gb, gg, gbt = B.snls_norm_backward(y, total, st, drop=0.25, rng=rng, site=3, grad_x=x)
    stats = st[:, B_ - 1, 0, H - 1, W - 300:].cpu()[:, None]
    (wx, _, _), (ex, _, _) = R.norm_backward(cut(y), cut(total), stats, None, None)
    _within(gx[end][:, None], wx, ex, "grad_x")
    assert torch.equal(gb[end].cpu() != 0, keep & (gx[end].cpu() != 0))
    for c in (0, C - 1):
        s = y[:, :, c].double().sum().item()
        # half a million chains of at most 300 roundings, whose errors add up like their number's root
        assert abs(float(gbt[c]) - s) < 300 * U * float(y[:, :, c].double().abs().sum())
    del gb, br, x, gx
    rp = dict(B=B_, T=1, C=C, H=H, W=W, HD=2, pairs=(3, 4, 5), theta=(100.0,) * 3)
    q, _ = B.snls_rotate(y, None, rp, q_out=total)
    far = dict(rp, B=1, H=1, W=300, row0=H - 1, col0=W - 300)
    got, src = q[end][None, None, :, None].cpu(), y[end][None, None, :, None].cpu()
    _within(got, R.rotate_video(src, torch.zeros(1, 1), far), R.rotate_bound(src, far, src.shape, 6000.0), "rotation")
    w = torch.randn(9, C, generator=g, device=dev)
    codes, scales = B.snls_project_pack(w)
    o = B.snls_project(y, codes, scales)
    want, err = R.project(y[end][None, None, :, None].cpu(), codes.cpu(), scales.cpu(), None, 1)
    _within(o[0][B_ - 1, 0, :, H - 1, W - 300:], want[0, 0, 0, :, 0], err[0, 0, 0, :, 0], "projection")
    del o, y, total, q
    torch.cuda.empty_cache()


# ------------------------------------------------------ as a layer uses them --

def test_training_layer_gradients(dev):
    """norm(x + dropout(branch)) -> rotation of q and k: the chain's gradients against autograd in 64 bits."""
    rp = dict(B=1, T=2, C=24, H=10, W=11, HD=2, pairs=(2, 2, 2), theta=(100.0, 100.0, 100.0))
    shp = B.video_shape(rp)
    g = _gen(12)
    x, br, gq, gk, gt = (torch.randn(shp, generator=g) for _ in range(5))
    gamma, beta = torch.randn(24, generator=g), torch.randn(24, generator=g)
    times = torch.tensor([[40, 41]])
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    more = dict(drop=0.2, rng=rng, site=3)
    y, total, stats = B.snls_norm(*_to(dev, x, gamma, beta), branch=br.to(dev), **more)
    qo, ko = B.snls_rotate(y, y, rp, times=times.to(dev))
    a, b = B.snls_rotate(*_to(dev, gq, gk), rp, times=times.to(dev), inverse=True)
    got = B.snls_norm_backward(a + b, total, stats, gamma.to(dev), grad_total=gt.to(dev), **more)
    leaves = [t.double().requires_grad_(True) for t in (x, br, gamma, beta)]
    tot = leaves[0] + torch.where(R.keep_mask(shp, RNG, 0.2, 3), leaves[1] / (1 - R.drop32(0.2)), 0.0)
    z = R.norm(tot, leaves[2], leaves[3], 1e-5)[0]
    wq = R.rotate_video(z, times, rp)
    assert float((qo.cpu().double() - wq.detach()).abs().max()) < 1e-5 and torch.equal(qo, ko)
    ((wq * gq.double()).sum() + (wq * gk.double()).sum() + (tot * gt.double()).sum()).backward()
    for v, leaf in zip(got, leaves):
        # some 50 roundings of sums of 24 (220 for the weights) terms: far below 1e-5 of the largest
        assert float((v.cpu().double() - leaf.grad).abs().max()) < 1e-5 * float(leaf.grad.abs().max())


def _attend64(q, k, v, inds, scale, HD):
    """Scores of the given neighbours (single pixels), their softmax and the weighted sum, in 64 bits."""
    B_, T, C, H, W = q.shape
    Ch = C // HD
    frame = inds[..., 0].long()
    hh = torch.arange(H).view(1, 1, 1, H, 1, 1)
    ww = torch.arange(W).view(1, 1, 1, 1, W, 1)
    bb = torch.arange(B_).view(B_, 1, 1, 1, 1, 1)
    hd = torch.arange(HD).view(1, HD, 1, 1, 1, 1)
    y, x = hh + inds[..., 1].double(), ww + inds[..., 2].double()
    ok = (frame >= 0) & (frame < T)

    def read(z):
        z = z.view(B_, T, HD, Ch, H, W).permute(0, 2, 1, 4, 5, 3)  # B HD T H W Ch
        out = 0
        for cy in (0, 1):
            for cx in (0, 1):
                Y, X = y.floor().long() + cy, x.floor().long() + cx
                wy = (y - y.floor()) if cy else 1 - (y - y.floor())
                wx = (x - x.floor()) if cx else 1 - (x - x.floor())
                on = ok & (Y >= 0) & (Y < H) & (X >= 0) & (X < W)
                tap = z[bb, hd, frame.clamp(0, T - 1), Y.clamp(0, H - 1), X.clamp(0, W - 1)]
                out = out + tap * (wy * wx * on)[..., None]
        return out

    d = (q.view(B_, T, HD, Ch, H, W).permute(0, 2, 1, 4, 5, 3)[..., None, :] * read(k)).sum(-1)
    logits = torch.where(ok, scale * d, torch.full_like(d, -1e30))
    out = (torch.softmax(logits, -1)[..., None] * read(v)).sum(-2)  # B HD T H W Ch
    return out.permute(0, 2, 1, 5, 3, 4).reshape(B_, T, C, H, W)


def test_training_layer_with_the_attention(dev):
    """Residual sum with dropout, norm, rotation, search, aggregation, a second dropout and norm, and back: the
    gradients against autograd in 64 bits at the neighbours that the search chose."""
    p = small_params(T=3, C=16, H=13, W=14, HD=2, ws=5, wt=1, ps=1, k=6)
    rp = dict(B=1, T=3, C=16, H=13, W=14, HD=2, pairs=(1, 1, 2), theta=(100.0, 50.0, 50.0), interleaved=True)
    shp, scale, drop = B.video_shape(p), 0.3, 0.25
    g = _gen(77)
    x, br, go = (torch.randn(shp, generator=g) for _ in range(3))
    gamma, beta, gamma2 = (1 + 0.3 * torch.randn(16, generator=g) for _ in range(3))
    flows = 1.3 * torch.randn(B.flow_shape(p), generator=g)
    times = torch.tensor([[70, 71, 72]])
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    xd, bd, gd, td, fd = _to(dev, x, br, go, times, flows)
    y, total, st = B.snls_norm(xd, gamma.to(dev), beta.to(dev), branch=bd, drop=drop, rng=rng, site=1)
    q, k = B.snls_rotate(y, y, rp, times=td)
    d, i = B.snls_search(q, k, fd, p)
    o = B.snls_aggregate(y, d, i, p, scale)
    y2, total2, st2 = B.snls_norm(total, gamma2.to(dev), branch=o, drop=drop, rng=rng, site=2)
    # back
    gt2, go_o, gg2, _ = B.snls_norm_backward(gd, total2, st2, gamma2.to(dev), drop=drop, rng=rng, site=2)
    gq, gk, gv, _ = B.snls_backward(q, k, y, fd, d, i, go_o, p, scale)
    a, b = B.snls_rotate(gq, gk, rp, times=td, inverse=True)
    gx, gb, gg, gbt = B.snls_norm_backward(a + b + gv, total, st, gamma.to(dev), grad_total=gt2, drop=drop, rng=rng,
                                           site=1)
    leaves = [t.double().requires_grad_(True) for t in (x, br, gamma, beta, gamma2)]
    f = 1 / (1 - R.drop32(drop))
    tot = leaves[0] + torch.where(R.keep_mask(shp, RNG, drop, 1), leaves[1] * f, 0.0)
    z = R.norm(tot, leaves[2], leaves[3], 1e-5)[0]
    qq = R.rotate_video(z, times, rp)
    out = _attend64(qq, qq, z, i.cpu(), scale, 2)
    # (the forward pass: some 100 roundings of values of up to 5)
    assert float((o.cpu().double() - out.detach()).abs().max()) < 100 * U * 5
    tot2 = tot + torch.where(R.keep_mask(shp, RNG, drop, 2), out * f, 0.0)
    (R.norm(tot2, leaves[4], None, 1e-5)[0] * go.double()).sum().backward()
    for v, leaf in zip((gx, gb, gg, gbt, gg2), leaves):
        # a few hundred roundings, of sums whose parts are up to some ten times the result: below 1e-4 of the largest
        assert float((v.cpu().double() - leaf.grad).abs().max()) < 1e-4 * float(leaf.grad.abs().max())


def _stream_state(dev, seed):
    g = torch.Generator(device=dev).manual_seed(seed)
    C, H, W, HD = 32, 21, 26, 2
    cp = dict(B=1, slots=2, C=C, H=H, W=W, HD=HD, block=8)
    rp = dict(B=1, T=1, C=C, H=H, W=W, HD=HD, pairs=(2, 3, 3), theta=(1000.0, 100.0, 100.0))
    w = torch.randn(3 * C, C, generator=g, device=dev) / math.sqrt(C)
    wo = torch.randn(C, C, generator=g, device=dev) / math.sqrt(C)
    return dict(cp=cp, rp=rp, x=torch.randn(1, 1, C, H, W, generator=g, device=dev), w=w, wo=wo,
                packed=B.snls_project_pack(w), packed_o=B.snls_project_pack(wo), cache=B.cache_alloc(cp, dev),
                ages=torch.tensor([[0, -1]], dtype=torch.int32, device=dev),
                slot=torch.zeros(1, dtype=torch.int32, device=dev), times=torch.tensor([[500]], device=dev),
                gamma=torch.rand(C, generator=g, device=dev) + 0.5)


def _stream_step(s):
    """One frame of a stream: norm, q k v, rotation, into the cache, attention, output projection, residual norm."""
    cp = s["cp"]
    y, _, _ = B.snls_norm(s["x"], s["gamma"])
    qkv = B.snls_project(y, *s["packed"], parts=3)
    q, k = B.snls_rotate(qkv[0], qkv[1], s["rp"], times=s["times"])
    frame = (cp["B"], cp["C"], cp["H"], cp["W"])
    B.snls_cache_store(k.view(frame), qkv[2].view(frame), s["slot"], cp, s["cache"])
    o = B.snls_cache_attend(q.view(frame), None, s["ages"], s["cache"], cp, 3, 0.25)
    branch = B.snls_project(o.view_as(s["x"]), *s["packed_o"])[0]
    y2, total, _ = B.snls_norm(s["x"], s["gamma"], branch=branch)
    return y, qkv, q, k, o, branch, y2, total


def test_stream_of_calls_and_its_graph(dev):
    s = _stream_state(dev, 5)
    y, qkv, q, k, o, branch, y2, total = _stream_step(s)
    cpu = lambda t: t.cpu()  # noqa: E731
    wy, _, _ = R.norm(cpu(s["x"]).double(), cpu(s["gamma"]), None, 1e-5)
    _within(y, wy, R.norm_bound(cpu(s["x"]).double(), cpu(s["gamma"]), None, 1e-5, torch.zeros_like(wy))[0], "norm")
    want, err = R.project(cpu(y), cpu(s["packed"][0]), cpu(s["packed"][1]), None, 3)
    _within(qkv, want, err, "q, k, v")
    for got, x in ((q, qkv[0]), (k, qkv[1])):
        _within(got, R.rotate_video(cpu(x), cpu(s["times"]), s["rp"]),
                R.rotate_bound(cpu(x), s["rp"], x.shape, 600.0), "rotation")
    want, err = R.project(cpu(o.view_as(s["x"])), cpu(s["packed_o"][0]), cpu(s["packed_o"][1]), None, 1)
    _within(branch, want[0], err[0], "output projection")
    t64 = cpu(s["x"]).double() + cpu(branch).double()
    _within(total, t64, U * t64.abs(), "residual")
    # eager results on three frames, then the same through one captured graph
    frames = [torch.randn_like(s["x"]) for _ in range(3)]
    eager = []
    for i, f in enumerate(frames):
        s["x"].copy_(f)
        s["times"].fill_(500 + i)
        eager.append([t.clone() for t in _stream_step(s)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _stream_step(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _stream_step(s)
    for i in (0, 1, 2, 0, 2):
        s["x"].copy_(frames[i])
        s["times"].fill_(500 + i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager[i]))


def test_training_step_in_a_graph_draws_new_masks(dev):
    shape = (1, 2, 32, 19, 23)
    x, br, gy, gt = (torch.randn(shape, device=dev) for _ in range(4))
    gamma = torch.rand(32, device=dev)
    rng = torch.tensor([11, 0], dtype=torch.int64, device=dev)

    def step():
        y, total, stats = B.snls_norm(x, gamma, branch=br, drop=0.4, rng=rng, site=2)
        grads = B.snls_norm_backward(gy, total, stats, gamma, grad_total=gt, drop=0.4, rng=rng, site=2)
        extra = B.snls_dropout(y, rng, 0.1, site=3, residual=x)
        return (y, total, stats) + grads + (extra,)

    eager = []
    for i in range(3):
        rng[1] = i
        eager.append([t.clone() for t in step()])
    assert not torch.equal(eager[0][1], eager[1][1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in (0, 1, 2, 1):
        rng[1] = i
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager[i]))


def test_memory_of_calls_on_another_stream(dev):
    shape = (1, 2, 32, 40, 41)
    g = torch.Generator(device=dev).manual_seed(3)
    x, gy = (torch.randn(shape, generator=g, device=dev) for _ in range(2))
    rp = dict(B=1, T=2, C=32, H=40, W=41, HD=1, pairs=(4, 6, 6), theta=(100.0,) * 3)
    rng = torch.tensor([1, 2], dtype=torch.int64, device=dev)
    codes, scales = B.snls_project_pack(torch.randn(64, 32, generator=g, device=dev))
    _, _, st = B.snls_norm(x)
    calls = [lambda **kw: B.snls_norm(x, branch=gy, **kw), lambda **kw: B.snls_norm_backward(gy, x, st, **kw),
             lambda **kw: B.snls_dropout(x, rng, 0.5, **kw), lambda **kw: B.snls_rotate(x, gy, rp, **kw),
             lambda **kw: B.snls_project(x, codes, scales, parts=2, **kw),
             lambda **kw: B.snls_project_pack(x.view(-1, 41), **kw)]
    flat = lambda o: [o] if isinstance(o, torch.Tensor) else list(o)  # noqa: E731
    side = torch.cuda.Stream()
    for call in calls:
        want = [t.clone() for t in flat(call())]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        outs = flat(call(stream=side))
        held = [(t.data_ptr(), t.numel()) for t in outs]
        del outs
        fresh = [torch.full((n,), float("nan"), device=dev) for _, n in held]
        assert not side.query()
        assert not {t.data_ptr() for t in fresh} & {at for at, _ in held}
        torch.cuda.synchronize()
        del fresh
        outs = flat(call(stream=side))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_misaligned_buffers(dev):
    """4-byte aligned, not more: views one element into their storage."""
    g = _gen(31)

    def off(t):
        s = torch.empty(t.numel() + 1, device=dev)[1:].view(t.shape)
        return s.copy_(t)

    for shape in ((1, 1, 48, 8, 16), (40, 64)):
        x, br = torch.randn(shape, generator=g).to(dev), torch.randn(shape, generator=g).to(dev)
        gamma = torch.randn(shape[-3] if len(shape) > 2 else 64, generator=g).to(dev)
        rng = torch.tensor([1, 2], dtype=torch.int64, device=dev)
        a = B.snls_norm(x, gamma, branch=br, drop=0.5, rng=rng)
        b = B.snls_norm(off(x), off(gamma), branch=off(br), drop=0.5, rng=rng, y=off(x), total=off(x))
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        ga = B.snls_norm_backward(br, a[1], a[2], gamma, grad_total=x)
        gb = B.snls_norm_backward(off(br), off(a[1]), off(a[2]), off(gamma), grad_total=off(x), grad_x=off(x))
        assert all(torch.equal(p, q) for p, q in zip(ga, gb))
        assert torch.equal(B.snls_dropout(x, rng, 0.5), B.snls_dropout(off(x), rng, 0.5, out=off(x)))
        cin = shape[-3] if len(shape) > 2 else 64
        codes, scales = B.snls_project_pack(torch.randn(33, cin, generator=g).to(dev))
        shifted = torch.empty(33 * cin + 1, dtype=torch.int8, device=dev)[1:].view(33, cin).copy_(codes)
        assert torch.equal(B.snls_project(x, codes, scales), B.snls_project(off(x), shifted, off(scales)))
    rp = dict(B=1, T=1, C=48, H=8, W=16, HD=1, pairs=(4, 6, 6), theta=(100.0,) * 3)
    x = torch.randn(1, 1, 48, 8, 16, generator=g).to(dev)
    assert torch.equal(B.snls_rotate(x, None, rp)[0], B.snls_rotate(off(x), None, rp, q_out=off(x))[0])


def test_the_binding_refuses(dev):
    x, tok = torch.zeros(1, 1, 8, 4, 4, device=dev), torch.zeros(3, 8, device=dev)
    rng = torch.tensor([1, 2], dtype=torch.int64, device=dev)
    rp = dict(B=1, T=1, C=8, H=4, W=4, HD=1, pairs=(1, 1, 1), theta=(10.0,) * 3)
    codes, scales = B.snls_project_pack(torch.ones(6, 8, device=dev))
    bad = [
        lambda: B.snls_norm(x.transpose(3, 4)[..., :2]), lambda: B.snls_norm(x.double()), lambda: B.snls_norm(x[0, 0, 0, 0]),
        lambda: B.snls_norm(x, gamma=torch.zeros(4, device=dev)), lambda: B.snls_norm(x, branch=tok),
        lambda: B.snls_norm(x, total=x), lambda: B.snls_norm(x, branch=x, drop=0.5),
        lambda: B.snls_norm(x, branch=x, drop=0.5, rng=torch.zeros(2, device=dev)),
        lambda: B.snls_norm_backward(x, x, torch.zeros(2, 1, 1, 4, device=dev)),
        lambda: B.snls_dropout(x, None, 0.5), lambda: B.snls_dropout(x, rng[:1], 0.5),
        lambda: B.snls_rotate(x, None, dict(rp, C=16)), lambda: B.snls_rotate(x, None, rp, k_out=x),
        lambda: B.snls_rotate(x, None, rp, times=torch.zeros(1, 1, dtype=torch.int32, device=dev)),
        lambda: B.snls_rotate(x, None, dict(rp, pairs=(1, 1))),
        lambda: B.snls_rotate_points(tok, torch.zeros(3, 3, device=dev), rp),
        lambda: B.snls_rotate_points(tok, torch.zeros(2, 3, dtype=torch.int32, device=dev), rp),
        lambda: B.snls_project(x, codes, scales, parts=4), lambda: B.snls_project(x, codes.float(), scales),
        lambda: B.snls_project(torch.zeros(3, 9, device=dev), codes, scales), lambda: B.snls_project(x, codes, scales[:5]),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: B.snls_norm(x, eps=-1.0), lambda: B.snls_norm(x, drop=0.5, rng=rng),
              lambda: B.snls_dropout(x, rng, 1.0), lambda: B.snls_rotate(x, None, dict(rp, pairs=(3, 1, 1)))):
        with pytest.raises(B.SnlsError):
            f()
