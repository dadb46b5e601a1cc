"""Sums over pixels and over channels of the norm and its gradients: their
rounding."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import layer64 as R

pytestmark = pytest.mark.gpu
U = R.U


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


# one tile or group of rows and more than a workgroup takes, of every way that the gradients are cut
SUMS = [(1, 1, 8, 5, 103), (2, 1, 48, 40, 41), (1, 1, 128, 16, 33), (4, 1, 48, 271, 483), (1, 5, 20, 256, 272),
        (1, 2, 192, 15, 17), (1, 1, 256, 8, 32), (5, 1, 192, 96, 97), (5, 1, 160, 96, 96),
        (1, 1, 300, 9, 32), (1, 1, 512, 8, 16), (3, 1, 384, 80, 81), (4, 1, 400, 72, 64),
        (2, 1, 600, 7, 9), (300, 2050), (65, 48), (20000, 48), (9000, 100), (33, 256), (9001, 256), (5000, 1000), (2500, 1024)]


@pytest.mark.parametrize("shape", SUMS, ids=str)
def test_gradients_of_the_weights_are_summed_in_64_bits(dev, shape):
    """With a mean of 0, an rstd of 1 and whole numbers every term is a whole number below 2^24 (exact in fp32), and
    every partial sum one below 2^53 (exact in 64 bits): what is left is one rounding of the whole sum."""
    g = torch.Generator(device=dev).manual_seed(sum(shape))
    C = shape[1] if len(shape) == 2 else shape[-3]
    gy = torch.randint(-2 ** 21, 2 ** 22, shape, generator=g, device=dev).float()
    total = torch.randint(-3, 4, shape, generator=g, device=dev).float()
    px = shape[:1] if len(shape) == 2 else shape[:2] + shape[3:]
    stats = torch.stack([torch.zeros(px, device=dev), torch.ones(px, device=dev)])
    gamma = torch.rand(C, generator=g, device=dev)
    rng = torch.tensor([3, 4], dtype=torch.int64, device=dev)
    _, _, gg, gb = B.snls_norm_backward(gy, total, stats, gamma, grad_total=total, drop=0.25, rng=rng)
    channels = [d for d in range(len(shape)) if d != (1 if len(shape) == 2 else 2)]
    assert torch.equal(gg, (gy.double() * total.double()).sum(channels).float())
    assert torch.equal(gb, gy.double().sum(channels).float())


# more channels than registers hold: tokens and frames
WIDE = [(3, 40000), (70, 2100), (2, 65535), (1, 2, 20000, 2, 3), (1, 1, 600, 8, 9)]


@pytest.mark.parametrize("shape", WIDE, ids=str)
def test_sums_of_many_channels(dev, shape):
    """Values far from zero, whose sum in fp32 would be off by some hundred roundings.  The sums being in 64 bits the
    mean has one rounding; a difference from it has that, and one of its own; the variance one; rstd three."""
    g = torch.Generator().manual_seed(shape[1])
    C = shape[1] if len(shape) == 2 else shape[2]
    x = torch.randn(shape, generator=g) + 700
    y, _, stats = B.snls_norm(x.to(dev), eps=1e-3)
    z = R.rows(x.double())
    wy, mean, rstd = R.norm(x.double(), None, None, 1e-3)
    dm = U * mean.abs() * (1 + 2.0 ** -12)
    d = (z - mean[..., None]).abs()
    dd = dm[..., None] + U * d * (1 + 2.0 ** -12)
    var = (d * d).mean(-1)
    dvar = (2 * d * dd + dd * dd).mean(-1) + 2 * U * (var + 1e-3)
    low = var + 1e-3 - dvar
    dr = 1 / torch.sqrt(low) - rstd + 3 * U / torch.sqrt(low)
    dy = (d + dd) * dr[..., None] + dd * rstd[..., None] + 3 * U * d * rstd[..., None]
    assert bool(((stats[0].cpu().double() - mean).abs() <= dm).all())
    assert bool(((stats[1].cpu().double() - rstd).abs() <= dr).all())
    assert bool(((R.rows(y.cpu().double()) - R.rows(wy)).abs() <= dy).all())


@pytest.mark.parametrize("shape", WIDE, ids=str)
def test_gradient_sums_of_many_channels(dev, shape):
    """A gradient whose mean is far larger than its spread.  Its mean over the channels in 64 bits: one rounding, and
    that of grad_y * gamma; the mean of the products with xh: two of xh, that, and one; then five of the rest."""
    g = torch.Generator().manual_seed(shape[1] + 1)
    C = shape[1] if len(shape) == 2 else shape[2]
    total, gy = torch.randn(shape, generator=g), torch.randn(shape, generator=g) + 700
    gamma = torch.rand(C, generator=g) + 0.5
    _, mean, rstd = R.norm(total.double(), None, None, 1e-3)
    stats = torch.stack([mean, rstd]).float()
    gx, _, _, _ = B.snls_norm_backward(gy.to(dev), total.to(dev), stats.to(dev), gamma.to(dev))
    (want, _, _), _ = R.norm_backward(gy, total, stats, gamma, None)
    m, r = stats[0].double()[..., None], stats[1].double()[..., None]
    xh, f = (R.rows(total.double()) - m) * r, R.rows(gy.double()) * gamma.double()
    mg, mgx = f.mean(-1, keepdim=True).abs(), (f * xh).mean(-1, keepdim=True).abs()
    dmg = U * f.abs().mean(-1, keepdim=True) + U * mg
    dmgx = 3 * U * (f * xh).abs().mean(-1, keepdim=True) + U * mgx
    size = f.abs() + mg + xh.abs() * mgx
    err = r * (U * f.abs() + dmg + xh.abs() * dmgx + 2 * U * xh.abs() * mgx + 5 * U * size) * (1 + 2.0 ** -12)
    assert bool(((R.rows(gx.cpu().double()) - R.rows(want)).abs() <= err).all())
