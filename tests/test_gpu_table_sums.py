"""The bias table's gradient holds its sums in 64 bits to the end.

Bound: an entry's n gradients are exact in 64 bits; in any order their sum is
off by at most n * 2^-53 * sum |g|, and one rounding to fp32 follows, half a
step: 2^-24 relative (2^-150 below the normal numbers).  Sums in fp32, also of
a share of the gradients, are off by up to 2^-24 of that share's sum and pass
the bound where the shares cancel; the tests check that on the CPU."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from workloads import small_params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _bound(ref, cnt, mag):
    return 2.0 ** -24 * ref.abs() + cnt * 2.0 ** -53 * mag + 2.0 ** -150


CASES = [
    (dict(T=2, C=4, H=80, W=81, k=40, ws=7, ps=1), 0, []), (dict(T=3, H=60, W=61, HD=2, k=20, ws=5, ps=1), 1, [0.5, 2.0]),
    (dict(T=3, H=64, W=64, HD=4, k=30, ws=7, ps=1, dist_type=1), 1, [0.5 + i for i in range(8)]),
    (dict(B=2, T=2, C=9, H=20, W=21, HD=3, k=7, ps=1), 1, [1.0 + i for i in range(16)]),
]


def _inputs(p, kind, seed):
    g = torch.Generator().manual_seed(seed)
    shp = B.out_shape(p)
    inds = torch.empty(shp + (3,))
    inds[..., 0] = torch.randint(0, p["T"], shp, generator=g).float()
    inds[..., 1:] = 4.0 * torch.randn(shp + (2,), generator=g)
    grad = torch.randn(shp, generator=g)
    if kind != "plain":  # the first half of every head's gradients cancels the second but for small parts
        half = shp[3] // 2  # query rows
        grad = grad.abs() + 0.5
        grad[:, :, :, half:] = grad[:, :, :, half:].flip(3)
        inds[:, :, :, shp[3] - half:] = inds[:, :, :, :half].flip(3)
        grad[:, :, :, shp[3] - half:] = -grad[:, :, :, :half].flip(3) * (1 + 2.0 ** -20)
        if kind == "large":
            grad = grad.clamp(-2, 2) * 1.5e38
    return torch.randn(shp, generator=g), inds, grad


@pytest.mark.parametrize("kind", ["plain", "cancel", "large"])
@pytest.mark.parametrize("kw,radius,edges", CASES, ids=range(len(CASES)))
def test_sums(dev, kw, radius, edges, kind):
    p, bias = small_params(**kw), dict(radius=radius, edges=edges)
    d, inds, grad = _inputs(p, kind, 5)
    print("sums", p, kind, flush=True)
    got = B.snls_bias_backward(grad.to(dev), d.to(dev), inds.to(dev), p, bias).cpu()
    ref, cnt, mag = R.table_grad(grad, d, inds, p, bias, p["HD"])
    inside = ref.abs() < 3.4028234e38
    assert bool(inside.any())
    bound = _bound(ref, cnt, mag)
    assert bool(((got.double() - ref).abs() <= bound)[inside].all())
    if kind != "plain":  # sums of 512 shares in fp32 pass the bound
        hd, st, bh, bw, ok = R.bias_entries(inds, p, bias)
        nb = 2 * len(edges) + 1
        at = (((hd * (2 * radius + 1) + st) * nb + bh) * nb + bw).expand(grad.shape)
        n = grad.numel()
        share = (torch.arange(n) * 512 // n).view(grad.shape)
        part = torch.zeros(512 * ref.numel(), dtype=R.F64)
        sign = 1.0 if p["dist_type"] == 0 else -1.0
        part.index_put_(((share * ref.numel() + at)[ok],), sign * grad[ok].double(), accumulate=True)
        low = part.float().double().view(512, -1).sum(0).view(ref.shape)
        assert not bool(((low - ref).abs() <= bound)[inside].all())


def test_two_million_into_one_entry(dev):
    """All of one sign: the last place is right."""
    p, bias = small_params(T=2, C=4, H=160, W=160, k=40, ws=7, wt=1, ps=1), dict(radius=0, edges=[])
    shp = B.out_shape(p)
    grad = torch.rand(shp, device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    got = float(B.snls_bias_backward(grad, torch.zeros(shp, device=dev), torch.zeros(shp + (3,), device=dev), p, bias))
    want, n = float(grad.double().sum()), grad.numel()
    assert abs(got - want) <= 2.0 ** -24 * want + 2 * n * 2.0 ** -53 * want
