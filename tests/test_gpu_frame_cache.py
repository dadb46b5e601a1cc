"""The 8-bit frame cache and the attention over it on the GPU against the
plain 64-bit forms (tests/attention64.py).

Tolerances.  Stored codes and scales are exact.  Attention: with u = 2^-24, a
logit is scale times a bilinear sum of dot products of Ch terms plus a table
entry, computed in fp32: |error| <= (Ch + 16) u (scale * sum |q| * max |k| +
scale * max |table|) = delta; a weight's relative error is at most 2 delta plus
the roundings of exp (a few u), of the difference from the maximum (u times the
largest difference, at most 2 max |logit|) and of the sums (n cells, u each at
worst); the output, a mean of values with these weights, is off by at most
max |v| times that, plus its own n additions."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import attention64 as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _cp(**kw):
    c = dict(B=1, slots=3, C=32, H=16, W=17, HD=2, block=8)
    c.update(kw)
    return c


def _filled(cp, dev, seed=0, amp=1.0):
    """A cache with every slot stored by the library, and its values in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    cache = B.cache_alloc(cp, dev)
    for s in range(cp["slots"]):
        k, v = (amp * torch.randn(cp["B"], cp["C"], cp["H"], cp["W"], generator=g) for _ in range(2))
        B.snls_cache_store(k.to(dev), v.to(dev), torch.full((cp["B"],), s, dtype=torch.int32, device=dev), cp, cache)
    return cache, R.decoded(cache[0], cache[1].cpu(), cp), R.decoded(cache[2], cache[3].cpu(), cp)


def _tol(q, kv, vv, cp, ws, scale, biggest, table):
    Ch, n = cp["C"] // cp["HD"], cp["slots"] * ws * ws
    fin = lambda x: torch.where(x.isfinite(), x, torch.zeros((), dtype=x.dtype)).abs()  # noqa: E731
    qs = float(fin(q.double()).view(q.shape[0], cp["HD"], Ch).sum(-1).max())
    tmax = float(fin(table).max()) if table is not None and float(fin(table).max()) < 1e30 else 0.0
    delta = abs(scale) * (Ch + 16) * U * (qs * float(fin(kv).max()) + tmax)
    return float(fin(vv).max()) * (2 * delta + 4 * biggest * U + 2 * n * U + 32 * U)


def _check(dev, cp, ws, q, points, flows, ages, cache, kv, vv, scale, table=None, bias=None):
    ref, biggest = R.attend(q, points, flows, ages, kv, vv, cp, ws, scale, table, bias)
    to = lambda x: None if x is None else x.to(dev)  # noqa: E731
    got = B.snls_cache_attend_points(to(q), to(points), to(flows), to(ages), cache, cp, ws, scale, table=to(table),
                                     bias=bias)
    err = (got.cpu().double() - ref).abs().max()
    tol = _tol(q, kv, vv, cp, ws, scale, biggest, table)
    print("err %.2e tol %.2e" % (float(err), tol), flush=True)
    assert float(err) <= tol
    return got, ref, tol


def _points(cp, n, g):
    return torch.stack([torch.randint(0, m, (n,), generator=g) for m in (cp["B"], cp["H"], cp["W"])], 1).to(torch.int32)


# ------------------------------------------------------------------- store --

@pytest.mark.parametrize("kw", [dict(), dict(B=3, C=20, HD=1, H=1, W=1), dict(C=1, HD=1, H=9, W=40, block=16),
                                dict(C=130, HD=2, H=17, W=33, block=16, B=2), dict(C=256, HD=1, H=8, W=8),
                                dict(C=48, HD=3, H=31, W=95), dict(C=34, HD=2, H=40, W=7, slots=1)], ids=range(7))
def test_store_is_exact(dev, kw):
    """Values over e4m3's whole range and a wide range of block sizes: codes and scales equal the definition's; only
    the named slots are written."""
    cp = _cp(**kw)
    g = torch.Generator().manual_seed(7)
    shp = (cp["B"], cp["C"], cp["H"], cp["W"])
    k, v = (torch.randn(shp, generator=g) * torch.exp2(torch.randint(-14, 15, shp, generator=g).float())
            for _ in range(2))
    v = v * torch.exp2(10.0 * torch.randint(-8, 9, (cp["B"], 1, cp["H"], cp["W"]), generator=g).float())
    k[:, :, : cp["H"] // 2] = 0  # blocks of zeros
    slots = torch.randint(0, cp["slots"], (cp["B"],), generator=g).to(torch.int32)
    if cp["B"] > 1:
        slots[0], slots[1] = -1, cp["slots"]  # left as they were
    cache = B.cache_alloc(cp, dev)
    for t in (cache[0], cache[2]):
        t.view(torch.uint8).fill_(0x55)
    for t in (cache[1], cache[3]):
        t.fill_(-3.0)
    print("store", cp, flush=True)
    B.snls_cache_store(k.to(dev), v.to(dev), slots.to(dev), cp, cache)
    Ch = cp["C"] // cp["HD"]
    for src, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        rc, rs = R.e4m3(src.view(cp["B"], cp["HD"], Ch, cp["H"], cp["W"]), cp["block"])
        codes, scales = codes.cpu(), scales.cpu()
        for b in range(cp["B"]):
            for s in range(cp["slots"]):
                if s != int(slots[b]):
                    assert bool((codes[b, s].view(torch.uint8) == 0x55).all()) and bool((scales[b, s] == -3).all())
                    continue
                assert torch.equal(scales[b, s].double(), rs[b])
                assert torch.equal(codes[b, s][..., :Ch].float().double(), rc[b].permute(0, 2, 3, 1))
                assert bool((codes[b, s][..., Ch:].view(torch.uint8) == 0).all())


@pytest.mark.parametrize("C", [80, 96, 100, 112, 127, 129, 160, 191, 192, 200, 240, 255])
def test_store_wide_heads(dev, C):
    """Every number of 16-channel vectors a token can have, and numbers of channels that do not fill the last."""
    cp = _cp(C=C, HD=1, H=21, W=35, slots=2)
    g = torch.Generator().manual_seed(71)
    k, v = (torch.randn(1, C, 21, 35, generator=g) * torch.exp2(torch.randint(-9, 9, (1, C, 21, 35), generator=g).float())
            for _ in range(2))
    cache = B.cache_alloc(cp, dev)
    cache[0].view(torch.uint8).fill_(0x55)
    B.snls_cache_store(k.to(dev), v.to(dev), torch.ones(1, dtype=torch.int32, device=dev), cp, cache)
    for src, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        rc, rs = R.e4m3(src.view(1, 1, C, 21, 35), 8)
        assert torch.equal(scales[0, 1].cpu().double(), rs[0])
        assert torch.equal(codes[0, 1].cpu()[..., :C].float().double(), rc[0].permute(0, 2, 3, 1))
        assert bool((codes[0, 1].cpu()[..., C:].view(torch.uint8) == 0).all())
    assert bool((cache[0][0, 0].view(torch.uint8) == 0x55).all())


def test_store_not_finite(dev):
    """Infinities are held as +-448 times the scale of the finite values, NaN as NaN; they do not touch the scale."""
    cp = _cp(C=16, HD=1, H=9, W=10, slots=1)
    g = torch.Generator().manual_seed(1)
    k = torch.randn(1, 16, 9, 10, generator=g)
    clean = k.clone()
    for (c, y, x), val in {(0, 0, 0): float("inf"), (3, 2, 5): -float("inf"), (5, 4, 4): float("nan"),
                           (0, 8, 9): float("inf")}.items():
        k[0, c, y, x], clean[0, c, y, x] = val, 0.0
    v = torch.full((1, 16, 9, 10), float("nan"))  # nothing finite: scale 1
    cache = B.cache_alloc(cp, dev)
    B.snls_cache_store(k.to(dev), v.to(dev), torch.zeros(1, dtype=torch.int32, device=dev), cp, cache)
    rc, rs = R.e4m3(clean.view(1, 1, 16, 9, 10), 8)
    assert torch.equal(cache[1].cpu().double()[:, 0], rs)
    codes = cache[0].cpu().float()[0, 0, 0]
    assert codes[0, 0, 0] == 448 and codes[2, 5, 3] == -448 and codes[8, 9, 0] == 448 and codes[4, 4, 5].isnan()
    assert bool(cache[2].float().isnan().all()) and bool((cache[3] == 1).all())


# ------------------------------------------------------------------ attend --

ATTEND = [  # (cache, ws, points, bias edges or None, radius)
    (dict(), 3, 40, [0.5, 2.0], 1),
    (dict(C=16, HD=1, slots=1), 1, 7, None, 0),
    (dict(C=1, HD=1, H=1, W=1), 2, 3, [1.0], 0),
    (dict(C=20, HD=1, H=1, W=40, slots=2), 9, 33, [0.5, 1.0, 4.0], 2),
    (dict(B=2, C=96, HD=2, H=20, W=11, block=16, slots=2), 7, 30, None, 0),
    (dict(C=64, HD=1, H=33, W=20, slots=5), 9, 40, [0.5, 1.0, 2.0, 4.0, 8.0], 3),
    (dict(C=100, HD=1, H=12, W=30, slots=2), 5, 20, [2.0], 5),
    (dict(C=256, HD=1, H=18, W=18, slots=2), 8, 12, [2.0], 1),
    (dict(C=180, HD=1, H=18, W=18, slots=2), 15, 12, [2.0], 1),
    (dict(C=36, HD=3, H=31, W=29, slots=7), 15, 20, [float(i + 1) for i in range(10)], 3),
    (dict(C=32, HD=2, H=24, W=24, slots=19), 11, 6, [1.0, 3.0], 12),
]


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("kw,ws,n,edges,radius", ATTEND, ids=range(len(ATTEND)))
def test_attend(dev, kw, ws, n, edges, radius, dense):
    cp = _cp(**kw)
    g = torch.Generator().manual_seed(11)
    cache, kv, vv = _filled(cp, dev)
    bias = None if edges is None else dict(radius=radius, edges=edges)
    table = None if edges is None else torch.randn(B.bias_table_shape(bias, cp["HD"]), generator=g)
    scale = 1.0 / (cp["C"] // cp["HD"]) ** 0.5
    ages = torch.stack([torch.randperm(cp["slots"], generator=g) for _ in range(cp["B"])]).to(torch.int32)
    if cp["slots"] > 2:
        ages[0, 1] = -1
    # offsets: fractions, whole pixels, just below whole pixels, beyond the frame on every side
    fl = 4 * torch.randn(cp["B"], cp["slots"], 2, cp["H"], cp["W"], generator=g)
    kind = torch.randint(0, 8, fl.shape, generator=g)
    fl = torch.where(kind == 0, fl.round(), fl)
    fl = torch.where(kind == 1, torch.nextafter(fl.round(), torch.full_like(fl, -100.0)), fl)
    fl = torch.where(kind == 2, fl * 8, fl)
    print("attend", cp, ws, dense, flush=True)
    if not dense:
        points = _points(cp, n, g)
        q = 2 * torch.randn(n, cp["C"], generator=g)
        b, h, w = (points[:, j].long() for j in range(3))
        _check(dev, cp, ws, q, points, fl[b, :, :, h, w].contiguous(), ages, cache, kv, vv, scale, table, bias)
        return
    q = 2 * torch.randn(cp["B"], cp["C"], cp["H"], cp["W"], generator=g)
    to = lambda x: None if x is None else x.to(dev)  # noqa: E731
    got = B.snls_cache_attend(to(q), to(fl), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    again = B.snls_cache_attend(to(q), to(fl), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    assert torch.equal(got, again)
    points = _points(cp, 4 * n, g)  # some of the frame's pixels, its corners among them
    points[0], points[1] = torch.tensor([0, 0, 0]), torch.tensor([cp["B"] - 1, cp["H"] - 1, cp["W"] - 1])
    b, h, w = (points[:, j].long() for j in range(3))
    qp, fp = q[b, :, h, w].contiguous(), fl[b, :, :, h, w].contiguous()
    ref, biggest = R.attend(qp, points, fp, ages, kv, vv, cp, ws, scale, table, bias)
    tol = _tol(qp, kv, vv, cp, ws, scale, biggest, table)
    assert float((got.cpu().double()[b, :, h, w] - ref).abs().max()) <= tol
    # every pixel: the two forms are the same operator
    allp = torch.stack(torch.meshgrid(*(torch.arange(m) for m in (cp["B"], cp["H"], cp["W"])), indexing="ij"), -1)
    allp = allp.view(-1, 3).to(torch.int32)
    qa = q.permute(0, 2, 3, 1).reshape(-1, cp["C"]).contiguous()
    fa = fl.permute(0, 3, 4, 1, 2).reshape(-1, cp["slots"], 2).contiguous()
    pts = B.snls_cache_attend_points(to(qa), to(allp), to(fa), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    pts = pts.view(cp["B"], cp["H"], cp["W"], cp["C"]).permute(0, 3, 1, 2)
    tol = _tol(qa, kv, vv, cp, ws, scale, biggest, table)
    assert float((pts - got).abs().max()) <= 2 * tol


def _both(dev, cp, ws, q, flows, ages, cache, scale, table=None, bias=None):
    """The dense form, and the same through the list of all pixels, as (n, C) each."""
    to = lambda x: None if x is None else x.to(dev)  # noqa: E731
    a = B.snls_cache_attend(to(q), to(flows), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    allp = torch.stack(torch.meshgrid(*(torch.arange(m) for m in (cp["B"], cp["H"], cp["W"])), indexing="ij"), -1)
    allp = allp.view(-1, 3).to(torch.int32)
    qa = q.permute(0, 2, 3, 1).reshape(-1, cp["C"]).contiguous()
    fa = None if flows is None else flows.permute(0, 3, 4, 1, 2).reshape(-1, cp["slots"], 2).contiguous()
    b = B.snls_cache_attend_points(to(qa), to(allp), to(fa), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    return a.permute(0, 2, 3, 1).reshape(-1, cp["C"]).cpu(), b.cpu(), qa, allp, fa


def test_rows_with_nothing_to_attend(dev):
    """Empty slots, offsets out of reach or not finite, buckets masked with -inf, queries of infinities and NaN: zeros,
    also where the cache holds NaN; a table of the lowest value keeps the softmax."""
    cp = _cp(slots=2, H=10, W=20)
    cache, kv, vv = _filled(cp, dev)
    cache[0].view(torch.uint8)[:, 1] = 0x7F  # NaN
    cache[2].view(torch.uint8)[:, 1] = 0x7F
    g = torch.Generator().manual_seed(2)
    q = torch.randn(1, 32, 10, 20, generator=g)
    fl = torch.randn(1, 2, 2, 10, 20, generator=g)
    none, one = torch.tensor([[-1, -5]], dtype=torch.int32), torch.tensor([[4, -1]], dtype=torch.int32)
    bias = dict(radius=1, edges=[1.0])
    for what, flows, ages, table in (
            ("empty", fl, none, None), ("far", fl + 1e6, one, None), ("past the frame", fl + 40.0, one, None),
            ("nan", fl * float("nan"), one, None), ("inf", fl * float("inf"), one, None),
            ("masked", fl, one, torch.full((2, 3, 3, 3), -float("inf")))):
        a, b, *_ = _both(dev, cp, 5, q, flows, ages, cache, 0.25, table, bias if table is not None else None)
        assert bool((a == 0).all()) and bool((b == 0).all()), what
    for val in (float("nan"), float("inf")):
        qb = q.clone()
        qb[0, :16, 3, 4], qb[0, 5, 7, 8] = val, val  # head 0 of two pixels
        a, b, *_ = _both(dev, cp, 5, qb, fl, one, cache, 0.25)
        for o in (a, b):
            o = o.view(10, 20, 32)
            assert bool((o[3, 4, :16] == 0).all()) and bool((o[7, 8, :16] == 0).all()) and bool(o.isfinite().all())
            assert bool((o[3, 4, 16:] != 0).any())
    low = torch.full((2, 3, 3, 3), torch.finfo(torch.float32).min)
    for o in _both(dev, cp, 5, q, fl, one, cache, 1.0, low, bias)[:2]:  # the scores vanish beside it: a plain mean
        assert bool(o.isfinite().all()) and bool((o != 0).any())
        qz = torch.zeros_like(q)
        mean = _both(dev, cp, 5, qz, fl, one, cache, 1.0)[0]
        assert float((o - mean).abs().max()) <= 64 * U * float(vv[:, 0].abs().max())


def test_not_finite_tokens(dev):
    """A NaN key takes out the candidates that read it and no other; NaN values that only taps of weight 0 reach,
    and values outside the window, stay out of the result."""
    cp = _cp(slots=2, C=20, HD=1, H=14, W=15)
    cache, kv, vv = _filled(cp, dev)
    g = torch.Generator().manual_seed(3)
    k8, v8 = cache[0].view(torch.uint8), cache[2].view(torch.uint8)
    k8[0, 0, 0, 6, 7, 3] = 0x7F
    k8[0, 1, 0, 0, 0, 0] = 0x7F
    v8[0, 1, 0, 9, 9, :20] = 0x7F
    kv, vv = R.decoded(cache[0], cache[1].cpu(), cp), R.decoded(cache[2], cache[3].cpu(), cp)
    ages = torch.tensor([[1, 2]], dtype=torch.int32)
    fl = torch.randn(1, 2, 2, 14, 15, generator=g)
    fl[:, 1] = fl[:, 1].round()  # whole pixels: their neighbours' taps have weight 0
    q = torch.randn(1, 20, 14, 15, generator=g)
    a, b, qa, allp, fa = _both(dev, cp, 5, q, fl, ages, cache, 0.2)
    ref, biggest = R.attend(qa, allp, fa, ages, kv, vv, cp, 5, 0.2)
    tol = _tol(qa, kv, vv, cp, 5, 0.2, biggest, None)
    assert bool(ref.isnan().any()) and bool(ref.isfinite().any())
    for o in (a, b):
        assert torch.equal(o.isnan(), ref.isnan())
        fin = ref.isfinite()
        assert float((o.double() - ref)[fin].abs().max()) <= tol


def test_points_outside_and_repeated(dev):
    cp = _cp(B=2)
    cache, kv, vv = _filled(cp, dev)
    g = torch.Generator().manual_seed(4)
    pts = torch.tensor([[0, 3, 4], [2, 0, 0], [-1, 0, 0], [0, 16, 0], [0, 0, 17], [0, -1, 5], [1, 15, 16], [0, 3, 4],
                        [0, 2 ** 30, 2 ** 30], [-2 ** 31, 2 ** 31 - 1, 0]], dtype=torch.int32)
    q = torch.randn(10, 32, generator=g)
    q[7] = q[0]
    ages = torch.zeros(2, 3, dtype=torch.int32)
    got, _, _ = _check(dev, cp, 5, q, pts, None, ages, cache, kv, vv, 0.3)
    assert torch.equal(got[0], got[7])
    for i in (1, 2, 3, 4, 5, 8, 9):
        assert bool((got[i] == 0).all())
    empty = B.snls_cache_attend_points(q[:0].to(dev), pts[:0].to(dev), None, ages.to(dev), cache, cp, 5)
    assert empty.shape == (0, 32)


def test_extreme_logits(dev):
    """Logits of thousands (one candidate takes all) and features of 1e18: fp32's range is not left on the way."""
    cp = _cp(C=16, HD=1, H=12, W=12, slots=2)
    cache, kv, vv = _filled(cp, dev, amp=1e18)
    g = torch.Generator().manual_seed(5)
    pts = _points(cp, 20, g)
    q = torch.randn(20, 16, generator=g) * 1e-15
    ages = torch.zeros(1, 2, dtype=torch.int32)
    # whole-pixel offsets: no cancelling between taps; the tolerance's exponent grows with the logits
    got, ref, tol = _check(dev, cp, 5, q, pts, torch.randn(20, 2, 2, generator=g).round(), ages, cache, kv, vv, 1.0)
    assert bool(got.isfinite().all())


def test_large_cache(dev):
    """Codes beyond 2^32 bytes: the last slot is written and read where it lies."""
    cp = dict(B=1, slots=70, C=64, H=1024, W=1024, HD=1, block=8)
    codes, scales = B.cache_shapes(cp)
    assert torch.Size(codes).numel() > 1 << 32
    cache = tuple(torch.empty(s, device=dev, dtype=t) for s, t in ((codes, torch.float8_e4m3fn), (scales, torch.float32),
                                                                   (codes, torch.float8_e4m3fn), (scales, torch.float32)))
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn(1, 64, 1024, 1024, generator=g) for _ in range(2))
    print("large cache", flush=True)
    B.snls_cache_store(k.to(dev), v.to(dev), torch.tensor([69], dtype=torch.int32, device=dev), cp, cache)
    ages = torch.full((1, 70), -1, dtype=torch.int32)
    ages[0, 69] = 1
    one = dict(cp, slots=1)
    sub = tuple(t[:, 69:].contiguous().cpu() for t in cache)
    kv, vv = R.decoded(sub[0], sub[1], one), R.decoded(sub[2], sub[3], one)
    pts = torch.tensor([[0, 1023, 1023], [0, 0, 0], [0, 1000, 3], [0, 511, 700]], dtype=torch.int32)
    q = torch.randn(4, 64, generator=g)
    fl = torch.randn(4, 70, 2, generator=g)
    got = B.snls_cache_attend_points(q.to(dev), pts.to(dev), fl.to(dev), ages.to(dev), cache, cp, 9, 0.125)
    ref, big = R.attend(q, pts, fl[:, 69:].contiguous(), ages[:, 69:], kv, vv, one, 9, 0.125)
    assert float((got.cpu().double() - ref).abs().max()) <= _tol(q, kv, vv, one, 9, 0.125, big, None)


def test_stream_of_frames(dev):
    """As a program runs it: frame by frame through a ring of slots, two videos that start at different times, the
    chain in a graph replayed per frame; every frame against 64 bits on the frames' own rounded values."""
    cp = _cp(B=2, slots=3, C=24, HD=2, H=19, W=21)
    bias = dict(radius=3, edges=[0.5, 1.0, 3.0])
    g = torch.Generator().manual_seed(9)
    table = torch.randn(B.bias_table_shape(bias, 2), generator=g)
    cache = B.cache_alloc(cp, dev)
    shp = (2, 24, 19, 21)
    q, k, v = (torch.empty(shp, device=dev) for _ in range(3))
    fl = torch.empty(2, 3, 2, 19, 21, device=dev)
    ages = torch.full((2, 3), -1, dtype=torch.int32, device=dev)
    slots = torch.zeros(2, dtype=torch.int32, device=dev)
    out = torch.empty(shp, device=dev)
    tg = table.to(dev)

    def step():
        B.snls_cache_attend(q, fl, ages, cache, cp, 5, 0.3, table=tg, bias=bias, out=out)
        B.snls_cache_store(k, v, slots, cp, cache)

    for s in (-1,):  # the first launches outside the graph, leaving the cache as it is
        slots.fill_(s)
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = {}
    start = (0, 2)
    for t in range(7):
        frame = [torch.randn(shp, generator=g) for _ in range(3)]
        flow = 2 * torch.randn(2, 3, 2, 19, 21, generator=g)
        a = torch.full((2, 3), -1, dtype=torch.int32)
        for (b, s), (when, _, _) in held.items():
            a[b, s] = t - when
        sl = torch.tensor([t % 3 if t >= start[b] else -1 for b in range(2)], dtype=torch.int32)
        for dst, src in zip((q, k, v, fl, ages, slots), frame + [flow, a, sl]):
            dst.copy_(src)
        kv, vv = torch.zeros(2, 3, 2, 19, 21, 12, dtype=R.F64), torch.zeros(2, 3, 2, 19, 21, 12, dtype=R.F64)
        for (b, s), (_, kk, vvv) in held.items():
            kv[b, s], vv[b, s] = kk, vvv
        graph.replay()
        torch.cuda.synchronize()
        pts = _points(cp, 25, g)
        b, h, w = (pts[:, j].long() for j in range(3))
        qp, fp = frame[0][b, :, h, w].contiguous(), flow[b, :, :, h, w].contiguous()
        ref, big = R.attend(qp, pts, fp, a, kv, vv, cp, 5, 0.3, table, bias)
        tol = _tol(qp, kv, vv, cp, 5, 0.3, big, table)
        assert float((out.cpu().double()[b, :, h, w] - ref).abs().max()) <= tol, t
        assert t > 0 or bool((out == 0).all())
        for b in range(2):
            if int(sl[b]) >= 0:
                rc, rs = zip(*(R.e4m3(x[b:b + 1].view(1, 2, 12, 19, 21), 8) for x in frame[1:]))
                vals = [(c * s.repeat_interleave(8, 2)[:, :, :19].repeat_interleave(8, 3)[..., :21][:, :, None])
                        for c, s in zip(rc, rs)]
                held[(b, int(sl[b]))] = (t,) + tuple(x[0].permute(0, 2, 3, 1) for x in vals)


def test_side_stream_and_two_calls(dev):
    """Two calls at once on two streams with their own outputs."""
    cp = _cp(C=64, HD=2, H=40, W=41)
    cache, _, _ = _filled(cp, dev)
    g = torch.Generator(device=dev).manual_seed(1)
    ages = torch.zeros(1, 3, dtype=torch.int32, device=dev)
    qs = [torch.randn(1, 64, 40, 41, device=dev, generator=g) for _ in range(2)]
    want = [B.snls_cache_attend(x, None, ages, cache, cp, 7, 0.2) for x in qs]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(x) for x in qs]
    for x, o, s in zip(qs, outs, st):
        B.snls_cache_attend(x, None, ages, cache, cp, 7, 0.2, out=o, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


@pytest.mark.parametrize("C,HD,ws,slots", [(16, 1, 2, 5), (24, 1, 4, 1), (40, 1, 6, 2), (64, 1, 10, 4), (70, 1, 3, 3),
                                           (96, 1, 12, 2), (130, 1, 9, 2), (250, 1, 5, 4), (48, 3, 9, 3),
                                           (112, 1, 15, 2)], ids=str)
def test_long_lists_of_points(dev, C, HD, ws, slots):
    """Lists long enough for four lanes a point, for every grouping of channels and window width: the same as the dense
    form, sampled against 64 bits, with points outside the frame among them."""
    cp = _cp(B=2, C=C, HD=HD, H=47, W=45, slots=slots)
    g = torch.Generator().manual_seed(21)
    cache, kv, vv = _filled(cp, dev)
    bias = dict(radius=2, edges=[0.5, 2.0, 5.0])
    table = torch.randn(B.bias_table_shape(bias, HD), generator=g)
    ages = torch.randint(-1, 4, (2, slots), generator=g).to(torch.int32)
    ages[:, 0] = 1
    q = 2 * torch.randn(2, C, 47, 45, generator=g)
    fl = 3 * torch.randn(2, slots, 2, 47, 45, generator=g)
    scale = 1.0 / (C // HD) ** 0.5
    print("points", cp, ws, flush=True)
    a, b, qa, allp, fa = _both(dev, cp, ws, q, fl, ages, cache, scale, table, bias)
    pick = torch.randint(0, qa.shape[0], (24,), generator=g)
    ref, big = R.attend(qa[pick], allp[pick], fa[pick], ages, kv, vv, cp, ws, scale, table, bias)
    tol = _tol(qa, kv, vv, cp, ws, scale, big, table)
    assert float((a[pick].double() - ref).abs().max()) <= tol
    assert float((b[pick].double() - ref).abs().max()) <= tol
    assert float((a - b).abs().max()) <= 2 * tol
    bad = allp.clone()
    bad[5::7, 0] = 2
    bad[6::7, 1] = -3
    to = lambda x: x.to(dev)  # noqa: E731
    got = B.snls_cache_attend_points(to(qa), to(bad), to(fa), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    got = got.cpu()
    keep = torch.ones(len(bad), dtype=torch.bool)
    keep[5::7] = keep[6::7] = False
    assert bool((got[~keep] == 0).all()) and torch.equal(got[keep], b[keep])


def _sampled(dev, cp, ws, q, fl, ages, cache, kv, vv, scale, n, g, table=None, bias=None):
    """The dense form and n of its pixels in 64 bits."""
    to = lambda x: None if x is None else x.to(dev)  # noqa: E731
    got = B.snls_cache_attend(to(q), to(fl), to(ages), cache, cp, ws, scale, table=to(table), bias=bias)
    pts = _points(cp, n, g)
    pts[0], pts[1] = torch.tensor([0, 0, 0]), torch.tensor([cp["B"] - 1, cp["H"] - 1, cp["W"] - 1])
    b, h, w = (pts[:, j].long() for j in range(3))
    qp = q[b, :, h, w].contiguous()
    ref, big = R.attend(qp, pts, fl[b, :, :, h, w].contiguous(), ages, kv, vv, cp, ws, scale, table, bias)
    return got.cpu().double()[b, :, h, w], ref, big, qp, got


@pytest.mark.parametrize("C,ws,slots,block", [(32, 9, 2, 8), (48, 5, 3, 16), (64, 9, 1, 8), (64, 7, 2, 16),
                                              (96, 11, 2, 8), (120, 9, 2, 8)], ids=str)
@pytest.mark.parametrize("spread", [3.0, 40.0])
def test_boxes(dev, C, ws, slots, block, spread):
    """Offsets of neighbouring pixels that share a box of tokens (3 pixels apart) and that do not (40 pixels)."""
    cp = _cp(B=2, C=C, HD=1, H=101, W=94, slots=slots, block=block)
    g = torch.Generator().manual_seed(31)
    cache, kv, vv = _filled(cp, dev)
    bias = dict(radius=1, edges=[1.0, 4.0])
    table = torch.randn(B.bias_table_shape(bias, 1), generator=g)
    q = 2 * torch.randn(2, C, 101, 94, generator=g)
    fl = spread * torch.randn(2, slots, 2, 101, 94, generator=g)
    fl[:, :, :, 40:60] = 0.25  # narrow boxes, and wide ones beside them
    ages = torch.zeros(2, slots, dtype=torch.int32)
    scale = 1.0 / C ** 0.5
    print("boxes", cp, ws, spread, flush=True)
    got, ref, big, qp, whole = _sampled(dev, cp, ws, q, fl, ages, cache, kv, vv, scale, 40, g, table, bias)
    assert float((got - ref).abs().max()) <= _tol(qp, kv, vv, cp, ws, scale, big, table)
    # all pixels, against the vector units' form of the same operator
    _, pts, qa, _, _ = _both(dev, cp, ws, q, fl, ages, cache, scale, table, bias)
    pts = pts.view(2, 101, 94, C).permute(0, 3, 1, 2)
    assert float((pts - whole.cpu()).abs().max()) <= 2 * _tol(qa, kv, vv, cp, ws, scale, big, table)


def test_channels_of_very_different_size(dev):
    """Keys whose channels are up to 2^14 apart and queries the other way round, so that all count alike.  The two fp16
    parts of a query's channel are off by at most 2^-22 of it: with S = sum |q_c| max |k_c| per query, a logit is off by
    at most scale * ((C + 16) u + 2^-22) S."""
    C = 64
    cp = _cp(C=C, HD=1, H=40, W=41, slots=2)
    g = torch.Generator().manual_seed(41)
    amp = torch.exp2(-14.0 * torch.arange(C) / (C - 1)).view(1, C, 1, 1)
    cache = B.cache_alloc(cp, dev)
    for s in range(2):
        k, v = (torch.randn(1, C, 40, 41, generator=g) for _ in range(2))
        B.snls_cache_store((k * amp).to(dev), v.to(dev), torch.full((1,), s, dtype=torch.int32, device=dev), cp, cache)
    kv, vv = R.decoded(cache[0], cache[1].cpu(), cp), R.decoded(cache[2], cache[3].cpu(), cp)
    q = torch.randn(1, C, 40, 41, generator=g) / amp
    fl = torch.randn(1, 2, 2, 40, 41, generator=g)
    ages = torch.zeros(1, 2, dtype=torch.int32)
    got, ref, big, qp, _ = _sampled(dev, cp, 9, q, fl, ages, cache, kv, vv, 0.125, 60, g)
    S = float((qp.double().abs() * kv.abs().amax((0, 1, 2, 3, 4))).sum(1).max())
    delta = 0.125 * ((C + 16) * U + 2.0 ** -22) * S
    tol = float(vv.abs().max()) * (2 * delta + 4 * big * U + 2 * 162 * U + 32 * U)
    print("err %.2e tol %.2e" % (float((got - ref).abs().max()), tol))
    assert float((got - ref).abs().max()) <= tol


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4, 1e30])
def test_query_sizes(dev, size):
    """Queries far from 1 against keys far the other way; a NaN or infinite channel of one query stays with it."""
    cp = _cp(C=64, HD=1, H=30, W=31, slots=2)
    g = torch.Generator().manual_seed(51)
    cache, kv, vv = _filled(cp, dev, amp=1.0 / size)
    q = size * torch.randn(1, 64, 30, 31, generator=g)
    fl = torch.randn(1, 2, 2, 30, 31, generator=g)
    ages = torch.zeros(1, 2, dtype=torch.int32)
    got, ref, big, qp, whole = _sampled(dev, cp, 9, q, fl, ages, cache, kv, vv, 0.125, 40, g)
    assert float((got - ref).abs().max()) <= _tol(qp, kv, vv, cp, 9, 0.125, big, None)
    bad = q.clone()
    bad[0, 7, 10, 11], bad[0, 9, 20, 3], bad[0, :, 5, 5] = float("nan"), float("inf"), 0.0
    out = B.snls_cache_attend(bad.to(dev), fl.to(dev), ages.to(dev), cache, cp, 9, 0.125)
    keep = torch.ones(30, 31, dtype=torch.bool, device=dev)
    keep[10, 11] = keep[20, 3] = keep[5, 5] = False
    assert bool((out[0, :, 10, 11] == 0).all()) and bool((out[0, :, 20, 3] == 0).all())
    assert torch.equal(out[:, :, keep], whole[:, :, keep]) and bool((out[0, :, 5, 5] != 0).any())


@pytest.mark.parametrize("C,HD,ws", [(64, 2, 9), (64, 1, 9), (96, 1, 5), (256, 2, 7)])
def test_wide_heads_in_a_graph_and_beside_another_call(dev, C, HD, ws):
    """Heads whose scores come from the matrix cores: replays with new inputs, offsets that are not finite, tokens
    that are NaN and slots that hold nothing; the same call on another stream meanwhile."""
    cp = _cp(B=2, C=C, HD=HD, H=37, W=45, slots=3)
    gen = torch.Generator(device=dev).manual_seed(61)
    cache, _, _ = _filled(cp, dev)
    q = torch.randn(2, C, 37, 45, device=dev, generator=gen)
    fl = torch.empty(2, 3, 2, 37, 45, device=dev)
    ages = torch.tensor([[2, 1, 0], [0, -1, 5]], dtype=torch.int32, device=dev)
    scale = 1.0 / (C // HD) ** 0.5
    keys = cache[0].view(torch.uint8)
    keys[0, 0, :, 10, 10, 3] = 0x7F  # NaN
    keys[1, 1] = 0x7F  # a slot that holds no frame
    cache[2].view(torch.uint8)[1, 1] = 0x7F
    out, other = torch.empty_like(q), torch.empty_like(q)

    def step(to):
        return B.snls_cache_attend(q, fl, ages, cache, cp, ws, scale, out=to)

    def fresh():
        fl.normal_(generator=gen).mul_(3)
        fl[0, 1, 0, 5:9, 3], fl[0, 2, 1, 20, 7:30], fl[1, 0, 0, 30] = float("nan"), float("inf"), 1e6
        fl[1, 2, :, :8, :8] = -1e5  # windows outside the frame
        q.normal_(generator=gen)

    fresh()
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    side = torch.cuda.Stream()
    for _ in range(3):
        fresh()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(other)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other) and torch.equal(out, step(torch.empty_like(q)))
        assert bool(out.isfinite().all())
        # the points' form of the same pixels, by the vector units
        b, h, w = torch.meshgrid(torch.arange(2), torch.arange(37), torch.arange(45), indexing="ij")
        pts = torch.stack([b, h, w], -1).view(-1, 3).to(torch.int32).to(dev)
        qp = q.permute(0, 2, 3, 1).reshape(-1, C).contiguous()
        fp = fl.permute(0, 3, 4, 1, 2).reshape(-1, 3, 2).contiguous()
        got = B.snls_cache_attend_points(qp, pts, fp, ages, cache, cp, ws, scale).view(2, 37, 45, C)
        kv, vv = (torch.full((1,), x, dtype=R.F64) for x in (6.0, 6.0))  # |N(0,1)| of these sizes stays below 6
        tol = 2 * _tol(qp.cpu(), kv, vv, cp, ws, scale, 60.0, None)
        assert float((got.permute(0, 3, 1, 2) - out).abs().max()) <= tol
