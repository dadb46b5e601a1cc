"""Ways through the kernels that only larger calls take: several tiles, groups or
rows a workgroup, weights in two buffers, every instance of the projections."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import layer64 as R

pytestmark = pytest.mark.gpu
U = R.U
RNG = (-0x1234567890abcde, 77)


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _within(got, want, bound, what):
    off = (got.detach().cpu().double() - want).abs()
    over = off > bound
    assert not bool(over.any()) and not bool(off.isnan().any()), "%s: %d of %d out of bounds, worst %.3g over %.3g" % (
        what, int(over.sum()), over.numel(), float(off[over].max()), float(bound.expand_as(off)[over].min()))


# ------------------------------------------------------- the norm's gradients --

# more tiles (or groups of tokens) than workgroups: up to 128 channels more than 512 runs of 256 pixels (up to 32
# channels more than 1,024), up to 256 runs of 64, up to 512 runs of 32; 512 groups of 16 or 4 tokens
TURNS = [(1, 3, 48, 224, 228), (1, 3, 48, 221, 233), (1, 5, 20, 256, 272), (1, 5, 9, 255, 271), (1, 5, 192, 96, 97), (1, 5, 130, 96, 96),
         (1, 3, 384, 80, 81), (1, 3, 300, 72, 96), (1, 3, 500, 75, 77), (20000, 48), (9000, 100), (9001, 256),
         (5000, 1000), (2600, 1024)]


@pytest.mark.parametrize("shape", TURNS, ids=str)
def test_gradients_over_several_tiles_a_workgroup(dev, shape):
    g = torch.Generator().manual_seed(sum(shape))
    C = shape[1] if len(shape) == 2 else shape[2]
    total, gy, gt = torch.randn(shape, generator=g) + 0.5, torch.randn(shape, generator=g) + 0.25, torch.randn(shape, generator=g)
    gamma = torch.randn(C, generator=g)
    _, mean, rstd = R.norm(total.double(), None, None, 1e-5)
    stats = torch.stack([mean, rstd]).float()
    rng = torch.tensor(RNG, dtype=torch.int64, device=dev)
    gx, gb, gg, gbt = B.snls_norm_backward(gy.to(dev), total.to(dev), stats.to(dev), gamma.to(dev),
                                           grad_total=gt.to(dev), drop=0.3, rng=rng, site=4)
    (wx, wg, wb), (ex, _, _) = R.norm_backward(gy, total, stats, gamma, gt)
    _within(gx, wx, ex, "grad_x")
    # sums in 64 bits: two roundings of xh a term, the rounding of the result
    xh = (R.rows(total.double()) - stats[0].double()[..., None]) * stats[1].double()[..., None]
    size = (R.rows(gy.double()) * xh).abs().reshape(-1, C).sum(0)
    _within(gg, wg, (2 * U * size + U * wg.abs()) * (1 + 2.0 ** -12), "grad_gamma")
    _within(gbt, wb, U * wb.abs() * (1 + 2.0 ** -12), "grad_beta")
    keep = R.keep_mask(shape, RNG, 0.3, 4)
    f = 1 / (1 - R.drop32(0.3))
    _within(gb, torch.where(keep, wx * f, 0.0), torch.where(keep, (ex + 2 * U * wx.abs()) * f * (1 + 4 * U), 0.0), "grad_branch")


def test_gradients_of_the_weights_past_32_bits(dev):
    """4.4 thousand million elements: as in the smaller test of these sums, whole numbers leave one rounding."""
    shape = (2, 1, 68, 5700, 5700)
    if torch.cuda.mem_get_info()[0] < 80e9:
        pytest.skip("not enough memory")
    g = torch.Generator(device=dev).manual_seed(9)
    gy = torch.empty(shape, device=dev).random_(-2 ** 18, 2 ** 20, generator=g)
    total = torch.empty(shape, device=dev).random_(-3, 4, generator=g)
    px = shape[:2] + shape[3:]
    stats = torch.stack([torch.zeros(px, device=dev), torch.ones(px, device=dev)])
    gx, _, gg, gb = B.snls_norm_backward(gy, total, stats)
    del gx
    for c in range(shape[2]):
        a, b = gy[:, :, c].double(), total[:, :, c].double()
        assert float(gg[c]) == float((a * b).sum().float()) and float(gb[c]) == float(a.sum().float()), c
    del gy, total, stats, a, b
    torch.cuda.empty_cache()


# --------------------------------------- more tiles, tokens or heads than a grid --

def test_norm_over_more_tiles_than_a_grid(dev):
    """More than 2^21 runs of 128 pixels, and of 16 tokens: a pixel's result is that of a call on its rows alone."""
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("not enough memory")
    for W in (16512, 16511):  # planes that start a cache line, and that do not
        x = torch.randn(1, 1, 9, 16512, W, generator=torch.Generator(device=dev).manual_seed(W), device=dev)
        y, _, stats = B.snls_norm(x)
        for rows in (slice(0, 3), slice(16256, 16260), slice(16509, 16512)):
            want, _, st = B.snls_norm(x[..., rows, :].contiguous())
            assert torch.equal(y[..., rows, :], want) and torch.equal(stats[..., rows, :], st)
        del x, y, stats
    x = torch.randn(34_000_001, 5, generator=torch.Generator(device=dev).manual_seed(1), device=dev)
    y, _, stats = B.snls_norm(x)
    for rows in (slice(0, 50), slice(2 ** 25 - 20, 2 ** 25 + 20), slice(34_000_001 - 33, None)):
        want, _, st = B.snls_norm(x[rows].contiguous())
        assert torch.equal(y[rows], want) and torch.equal(stats[:, rows], st)
    del x, y, stats
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rp", [dict(B=30, T=20, C=16, H=3, W=6, HD=2, pairs=(1, 1, 1)),
                                dict(B=1, T=2, C=2300, H=3, W=7, HD=1, pairs=(2, 1, 3))], ids=["heads", "channels"])
def test_rotation_of_more_heads_and_channels_than_a_grid(dev, rp):
    rp = dict(rp, theta=(100.0, 50.0, 20.0))
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn(B.video_shape(rp), generator=g) for _ in range(2))
    times = torch.randint(0, 2000, (rp["B"], rp["T"]), generator=g)
    got = B.snls_rotate(q.to(dev), k.to(dev), rp, times=times.to(dev))
    for x, z in zip((q, k), got):
        _within(z, R.rotate_video(x, times, rp), R.rotate_bound(x, rp, x.shape, 2000.0), "rotation")


def test_rotation_of_more_tokens_than_a_grid(dev):
    rp = dict(B=3, T=1, C=16, H=50, W=60, HD=2, pairs=(1, 1, 1), theta=(100.0, 50.0, 20.0))
    g, n = torch.Generator().manual_seed(4), 700_001
    q = torch.randn(n, 16, generator=g)
    points = torch.stack([torch.randint(-1, m + 1, (n,), generator=g) for m in (3, 50, 60)], 1).to(torch.int32)
    times = torch.tensor([5, 600, 70])
    out = B.snls_rotate_points(q.to(dev), points.to(dev), rp, times=times.to(dev))
    _within(out, R.rotate_points(q, points, times, rp), R.rotate_bound(q, rp, q.shape, 700.0), "points")


# ------------------------------------------------------------ the projections --

# (shape of x, cout, parts)
ROUTES = [
    # runs of pixels, 1 to 6 steps of 32 channels, planes that start a cache line; whole and partial last steps
    ((1, 2, 32, 9, 32), 96, 3), ((1, 1, 16, 7, 64), 128, 1), ((2, 1, 64, 8, 20), 192, 3), ((1, 1, 96, 7, 32), 200, 1),
    ((1, 3, 80, 8, 12), 64, 2), ((1, 2, 128, 16, 14), 256, 4), ((2, 2, 112, 4, 24), 33, 1), ((1, 2, 192, 16, 20), 576, 3),
    ((1, 1, 160, 9, 96), 320, 1), ((1, 1, 176, 4, 8), 32, 1),
    # the same with several runs, and more of them than workgroups
    ((1, 5, 192, 152, 152), 576, 3), ((1, 1, 160, 480, 448), 64, 2), ((1, 1, 16, 1100, 1056), 32, 1),
    ((3, 1, 96, 200, 208), 96, 3), ((1, 3, 32, 304, 320), 64, 2), ((1, 2, 128, 304, 320), 160, 1),
    # a tile of weights after the other through two buffers, 7 to 16 steps, planes that start a line and that do not
    ((2, 1, 384, 128, 128), 384, 3), ((1, 1, 512, 130, 131), 520, 1), ((1, 1, 512, 128, 136), 520, 2), ((1, 1, 256, 150, 151), 700, 1),
    ((1, 1, 240, 160, 160), 640, 2),
    # the same with more groups of pixels than workgroups
    ((3, 1, 384, 152, 152), 384, 3), ((3, 1, 384, 151, 153), 384, 1), ((1, 3, 512, 150, 153), 130, 1), ((1, 1, 256, 264, 256), 288, 1),
    # rows of weights that do not start at 16 bytes: two buffers, and one with several groups a workgroup
    ((1, 1, 250, 300, 301), 700, 1), ((1, 1, 190, 256, 257), 640, 2), ((1, 3, 20, 300, 301), 48, 3), ((1, 2, 20, 304, 320), 100, 1),
    ((1, 1, 100, 300, 304), 1000, 4),
    # 1,001 channels, a tile of weights a buffer: 66,560 bytes of LDS
    ((1, 1, 1001, 256, 260), 96, 1), ((1, 1, 1001, 255, 261), 130, 2), ((66000, 1001), 96, 3),
    # no more than a group each of 385 to 512 channels
    ((1, 1, 512, 8, 16), 64, 1), ((1, 2, 400, 5, 9), 70, 2),
]


@pytest.mark.parametrize("case", ROUTES, ids=str)
def test_project_routes(dev, case):
    """Some pixels, the first and the last among them, within the bounds of the 64-bit form; all of them equal to what
    they give as tokens (frames only); nothing beside the output; the same again."""
    shape, cout, parts = case
    tokens = len(shape) == 2
    cin = shape[1] if tokens else shape[-3]
    g = torch.Generator(device=dev).manual_seed(cout + cin)
    x = torch.randn(shape, generator=g, device=dev)
    w = torch.randn(cout, cin, generator=g, device=dev)
    bias = torch.randn(cout, generator=g, device=dev)
    codes, scales = B.snls_project_pack(w)
    n = cout * (x.numel() // cin)
    room = torch.full((n + 64,), -7.5, device=dev)  # (its start is that of a cache line)
    tail = () if tokens else tuple(shape[-2:])
    out = room[:n].view((parts,) + (shape[:1] if tokens else shape[:-3]) + (cout // parts,) + tail)
    B.snls_project(x, codes, scales, bias=bias, parts=parts, out=out)
    assert bool((room[n:] == -7.5).all())
    pixels = 1 if tokens else shape[-2] * shape[-1]
    rows = x.view(-1, cin, pixels).transpose(1, 2).reshape(-1, cin)
    got = out.view(parts, -1, cout // parts, pixels).transpose(2, 3).reshape(parts, -1, cout // parts)
    total = rows.shape[0]
    some = torch.randint(0, total, (300,), generator=torch.Generator().manual_seed(1))
    some[:4], some[-4:] = torch.tensor([0, 1, 31, 32]).clamp(max=total - 1), torch.arange(total - 4, total)
    want, err = R.project(rows[some.to(dev)].cpu(), codes.cpu(), scales.cpu(), bias.cpu(), parts)
    _within(got[:, some.to(dev)], want, err, "project")
    if not tokens:
        assert torch.equal(got, B.snls_project(rows.contiguous(), codes, scales, bias=bias, parts=parts))
    assert torch.equal(out, B.snls_project(x, codes, scales, bias=bias, parts=parts))
