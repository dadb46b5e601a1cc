"""Attention over cached frames on the matrix cores holds 22 bits of a query.

The worst-case bounds of test_gpu_frame_cache.py are far above what roundings
do: these are independent.  A logit is a sum of Ch <= 128 products whose
partial sums stay within a few times the logits' size (2, as scale = 1 /
sqrt(Ch) and queries are 2 N(0, 1)); with u = 2^-24 for an operation, 2^-22
for a query's channel, its error is about sqrt(2 Ch) * u * 2 + 2^-22 * 2 < 3e-6
(one deviation), and the outputs, means over 81 candidates a slot of values up to max |v|,
move by less.  The bound, 1e-5 * max |v|, is several deviations above it.  Queries
rounded to fp16 alone (11 bits) move the logits 2^11 times as far: each test
checks on the CPU that this passes the bound."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from tests.test_gpu_frame_cache import _cp, _filled, _sampled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _run(dev, cp, ws, q, fl, cache, kv, vv, scale, g, table=None, bias=None, n=40):
    ages = torch.zeros(cp["B"], cp["slots"], dtype=torch.int32)
    seed = g.get_state()
    got, ref, _, qp, _ = _sampled(dev, cp, ws, q, fl, ages, cache, kv, vv, scale, n, g, table, bias)
    bound = 1e-5 * float(vv.abs().max())
    err = float((got - ref).abs().max())
    # the same pixels with the queries' low parts lost
    g.set_state(seed)
    top = q.abs().amax(1, keepdim=True)
    up = torch.exp2(14 - torch.floor(torch.log2(top)))
    lost = (q * up).half().float() / up
    pts = torch.stack([torch.randint(0, m, (n,), generator=g) for m in (cp["B"], cp["H"], cp["W"])], 1).to(torch.int32)
    pts[0], pts[1] = torch.tensor([0, 0, 0]), torch.tensor([cp["B"] - 1, cp["H"] - 1, cp["W"] - 1])
    b, h, w = (pts[:, j].long() for j in range(3))
    assert torch.equal(q[b, :, h, w], qp)
    half, _ = R.attend(lost[b, :, h, w].contiguous(), pts, fl[b, :, :, h, w].contiguous(), ages, kv, vv, cp, ws, scale,
                       table, bias)
    off = float((half - ref).abs().max())
    print("err %.2e bound %.2e, fp16 alone %.2e" % (err, bound, off), flush=True)
    assert off > bound
    assert err <= bound


@pytest.mark.parametrize("C,HD,ws,slots", [(32, 1, 9, 2), (64, 2, 9, 2), (48, 1, 5, 3), (64, 1, 9, 1), (64, 1, 7, 2),
                                           (96, 1, 11, 2), (120, 1, 9, 2), (128, 1, 5, 2), (80, 1, 9, 3)], ids=str)
def test_ordinary_inputs(dev, C, HD, ws, slots):
    cp = _cp(B=2, C=C, HD=HD, H=61, W=54, slots=slots)
    g = torch.Generator().manual_seed(31)
    cache, kv, vv = _filled(cp, dev)
    bias = dict(radius=1, edges=[1.0, 4.0])
    table = torch.randn(B.bias_table_shape(bias, HD), generator=g)
    q = 2 * torch.randn(2, C, 61, 54, generator=g)
    fl = 3.0 * torch.randn(2, slots, 2, 61, 54, generator=g)
    fl[:, :, :, 20:30] = 0.25
    _run(dev, cp, ws, q, fl, cache, kv, vv, (C // HD) ** -0.5, g, table, bias)


@pytest.mark.parametrize("C", [64, 128])
def test_channels_apart(dev, C):
    """Channels up to 2^12 apart in size, keys the other way round: the small channels' low parts count."""
    cp = _cp(C=C, HD=1, H=40, W=41, slots=2)
    g = torch.Generator().manual_seed(41)
    amp = torch.exp2(-12.0 * torch.arange(C) / (C - 1)).view(1, C, 1, 1)
    cache = B.cache_alloc(cp, dev)
    for s in range(2):
        k, v = (torch.randn(1, C, 40, 41, generator=g) for _ in range(2))
        B.snls_cache_store((k * amp).to(dev), v.to(dev), torch.full((1,), s, dtype=torch.int32, device=dev), cp, cache)
    kv, vv = R.decoded(cache[0], cache[1].cpu(), cp), R.decoded(cache[2], cache[3].cpu(), cp)
    q = torch.randn(1, C, 40, 41, generator=g) / amp
    fl = torch.randn(1, 2, 2, 40, 41, generator=g)
    _run(dev, cp, 9, q, fl, cache, kv, vv, C ** -0.5, g, n=60)


@pytest.mark.parametrize("C,HD,ws,slots", [(16, 1, 5, 2), (64, 1, 9, 2), (128, 1, 5, 1), (200, 1, 5, 2)], ids=str)
def test_extreme_logits(dev, C, HD, ws, slots):
    """Logits of hundreds and features of 1e18 through whole frames and long lists: the error grows with the logits, a
    logit L is off by about 2^-22 L and a weight by as much: 1e-5 max |v| per 16 of the largest logit."""
    from tests.test_gpu_frame_cache import _both
    cp = _cp(C=C, HD=HD, H=50, W=51, slots=slots)
    g = torch.Generator().manual_seed(5)
    cache, kv, vv = _filled(cp, dev, amp=1e18)
    q = 1e-16 * torch.randn(1, C, 50, 51, generator=g)
    fl = torch.randn(1, slots, 2, 50, 51, generator=g).round()
    ages = torch.zeros(1, slots, dtype=torch.int32)
    a, b, qa, allp, fa = _both(dev, cp, ws, q, fl, ages, cache, 1.0)
    pick = torch.randint(0, qa.shape[0], (30,), generator=g)
    ref, big = R.attend(qa[pick], allp[pick], fa[pick], ages, kv, vv, cp, ws, 1.0)
    assert big > 100
    bound = 1e-5 * float(vv.abs().max()) * max(big / 16, 1)
    for o in (a[pick], b[pick]):
        err = float((o.double() - ref).abs().max())
        print("err %.2e bound %.2e" % (err, bound), flush=True)
        assert err <= bound
