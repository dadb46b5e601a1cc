"""Sums over pixels and over channels of the norm and its gradients: their
rounding."""
import pytest
import torch

from paper_2309_16849_amd import snls as B

pytestmark = pytest.mark.gpu


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
