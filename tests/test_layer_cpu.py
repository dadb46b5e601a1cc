"""Refusals of the norm, dropout, rotary positions and 8-bit projections
(before any buffer or the device is touched), and checks of their plain 64-bit
forms."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2309_16849_amd as pkg
from paper_2309_16849_amd import snls as B
from tests import layer64 as R

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation first
BIG = 1 << 40
BAD, BEYOND = B.SNLS_ERR_INVALID_ARG, B.SNLS_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def _norm(C=8, frames=3, pixels=20, eps=1e-5, drop=0.0, site=0, size=None):
    return B.SnlsNormParams(size or ctypes.sizeof(B.SnlsNormParams), C, frames, pixels, eps, drop, site)


def _rot(**kw):
    rp = dict(B=1, T=2, C=16, H=5, W=6, HD=2, pairs=(1, 2, 1), theta=(100.0, 100.0, 100.0))
    rp.update(kw)
    return B.rotate_from_dict(rp)


def _proj(cin=8, cout=12, parts=3, frames=2, pixels=30, size=None):
    return B.SnlsProjectParams(size or ctypes.sizeof(B.SnlsProjectParams), cin, cout, parts, frames, pixels)


def test_struct_sizes():
    assert ctypes.sizeof(B.SnlsNormParams) == 40
    assert ctypes.sizeof(B.SnlsRotateParams) == 4 * 16
    assert ctypes.sizeof(B.SnlsProjectParams) == 32


def test_the_package_offers_them():
    for name in B.SYMBOLS:
        if name.startswith(("snls_norm", "snls_dropout", "snls_rotate", "snls_project")) and "workspace" not in name:
            assert getattr(pkg, name) is getattr(B, name)


BAD_NORM = [
    (dict(C=0), BAD), (dict(frames=-1), BAD), (dict(pixels=0), BAD), (dict(eps=-1e-5), BAD), (dict(eps=math.inf), BAD),
    (dict(eps=math.nan), BAD), (dict(drop=1.0), BAD), (dict(drop=-0.1), BAD), (dict(drop=math.nan), BAD),
    (dict(size=36), BAD), (dict(pixels=1 << 29), BEYOND), (dict(C=1 << 16), BEYOND), (dict(C=1 << 15, frames=1 << 20), BEYOND),
    (dict(frames=1 << 60, pixels=1 << 28), BEYOND),
]


@pytest.mark.parametrize("kw,want", BAD_NORM, ids=range(len(BAD_NORM)))
def test_norm_refuses_bad_sizes(lib, kw, want):
    prm = _norm(**kw)
    pn = ctypes.byref(prm)
    assert lib.snls_norm(FAKE, FAKE, FAKE, FAKE, FAKE, pn, FAKE, FAKE, FAKE, None) == want
    assert lib.snls_norm_backward(*[FAKE] * 6, pn, *[FAKE] * 5, BIG, None) == want
    assert lib.snls_norm_workspace_size(pn) == ctypes.c_size_t(-1).value


def test_norm_refuses_bad_arguments(lib):
    pn, dropped = ctypes.byref(_norm()), ctypes.byref(_norm(drop=0.5))
    call = lambda x=FAKE, br=FAKE, rng=FAKE, p=pn, tot=FAKE, y=FAKE: lib.snls_norm(  # noqa: E731
        x, br, rng, FAKE, FAKE, p, tot, y, FAKE, None)
    assert call(x=None) == BAD and call(y=None) == BAD and call(tot=None) == BAD and call(p=None) == BAD
    assert call(p=dropped, rng=None) == BAD and call(p=dropped, br=None) == BAD
    back = lambda a=FAKE, c=FAKE, d=FAKE, rng=FAKE, p=pn, gx=FAKE, gb=FAKE, gg=FAKE, gbt=FAKE, ws=FAKE, n=BIG: (  # noqa: E731
        lib.snls_norm_backward(a, FAKE, c, d, FAKE, rng, p, gx, gb, gg, gbt, ws, n, None))
    for kw in (dict(a=None), dict(c=None), dict(d=None), dict(gx=None), dict(gg=None), dict(gbt=None), dict(p=None),
               dict(p=dropped, rng=None), dict(p=dropped, gb=None)):
        assert back(**kw) == BAD, kw
    need = lib.snls_norm_workspace_size(pn)
    assert 0 < need < 1 << 30
    for ws, n in ((None, BIG), (FAKE, need - 1), (ctypes.c_void_p(0x1104), BIG)):
        assert back(ws=ws, n=n) == B.SNLS_ERR_WORKSPACE
    # nothing to do: no buffer is looked at
    empty = ctypes.byref(_norm(frames=0))
    assert call(x=None, br=None, p=empty, tot=None, y=None) == B.SNLS_OK
    assert back(a=None, c=None, d=None, p=empty, gx=None, gb=None, gg=None, gbt=None, ws=None) == B.SNLS_OK


def test_dropout_refuses(lib):
    call = lambda x=FAKE, r=None, rng=FAKE, n=100, d=0.5, out=FAKE: lib.snls_dropout(  # noqa: E731
        x, r, rng, n, d, 0, out, None)
    assert call(x=None) == BAD and call(rng=None) == BAD and call(out=None) == BAD and call(n=-1) == BAD
    for d in (1.0, -0.5, math.nan, math.inf):
        assert call(d=d) == BAD
    assert call(n=1 << 38) == BEYOND
    assert call(x=None, n=0, out=None) == B.SNLS_OK


BAD_ROT = [
    (dict(B=0), BAD), (dict(T=0), BAD), (dict(H=0), BAD), (dict(W=-1), BAD), (dict(HD=3), BAD), (dict(HD=0), BAD),
    (dict(pairs=(1, 2, 2)), BAD), (dict(pairs=(-1, 2, 1)), BAD), (dict(theta=(100.0, 0.0, 1.0)), BAD),
    (dict(theta=(math.inf, 1.0, 1.0)), BAD), (dict(theta=(1.0, 1.0, math.nan)), BAD), (dict(interleaved=2), BAD),
    (dict(C=1024, HD=1, pairs=(100, 20, 9)), BEYOND), (dict(H=1 << 15, W=1 << 15), BEYOND),
    (dict(C=1 << 20, HD=1, T=1 << 18, pairs=(1, 0, 0)), BEYOND),
    (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)), BAD),
]


@pytest.mark.parametrize("kw,want", BAD_ROT, ids=range(len(BAD_ROT)))
def test_rotate_refuses_bad_sizes(lib, kw, want):
    pr = ctypes.byref(_rot(**kw))
    assert lib.snls_rotate(FAKE, FAKE, FAKE, pr, 0, FAKE, FAKE, None) == want
    assert lib.snls_rotate_points(FAKE, FAKE, 5, FAKE, pr, 0, FAKE, None) == want


def test_rotate_refuses_bad_arguments(lib):
    pr = ctypes.byref(_rot())
    call = lambda q=FAKE, k=FAKE, p=pr, inv=0, qo=FAKE, ko=FAKE: lib.snls_rotate(q, k, None, p, inv, qo, ko, None)  # noqa: E731
    assert call(q=None) == BAD and call(qo=None) == BAD and call(k=None) == BAD and call(ko=None) == BAD
    assert call(inv=2) == BAD and call(inv=-1) == BAD and call(p=None) == BAD
    bad = _rot()
    bad.struct_size = 60
    assert call(p=ctypes.byref(bad)) == BAD
    pts = lambda q=FAKE, at=FAKE, n=3, p=pr, inv=0, out=FAKE: lib.snls_rotate_points(q, at, n, None, p, inv, out, None)  # noqa: E731
    assert pts(q=None) == BAD and pts(at=None) == BAD and pts(out=None) == BAD and pts(n=-1) == BAD
    assert pts(inv=3) == BAD and pts(p=None) == BAD and pts(n=1 << 40) == BEYOND
    assert pts(q=None, at=None, n=0, out=None) == B.SNLS_OK


BAD_PROJ = [
    (dict(cin=0), BAD), (dict(cout=0, parts=1), BAD), (dict(parts=0), BAD), (dict(parts=5), BAD), (dict(frames=-1), BAD),
    (dict(pixels=0), BAD), (dict(size=28), BAD), (dict(cin=1025), BEYOND), (dict(cout=3 << 15), BEYOND),
    (dict(pixels=1 << 25), BEYOND), (dict(frames=1 << 36), BEYOND), (dict(frames=1 << 50, pixels=1 << 20), BEYOND),
]


@pytest.mark.parametrize("kw,want", BAD_PROJ, ids=range(len(BAD_PROJ)))
def test_project_refuses_bad_sizes(lib, kw, want):
    pj = ctypes.byref(_proj(**kw))
    assert lib.snls_project(FAKE, FAKE, FAKE, FAKE, pj, FAKE, None) == want
    assert lib.snls_project_pack(FAKE, pj, FAKE, FAKE, None) == want


def test_project_refuses_bad_arguments(lib):
    pj = ctypes.byref(_proj())
    call = lambda x=FAKE, w=FAKE, s=FAKE, p=pj, out=FAKE: lib.snls_project(x, w, s, None, p, out, None)  # noqa: E731
    assert call(x=None) == BAD and call(w=None) == BAD and call(s=None) == BAD and call(out=None) == BAD
    assert call(p=None) == BAD
    for i in range(3):
        a = [FAKE] * 3
        a[i] = None
        assert lib.snls_project_pack(a[0], pj, a[1], a[2], None) == BAD
    assert lib.snls_project_pack(FAKE, None, FAKE, FAKE, None) == BAD
    assert call(x=None, p=ctypes.byref(_proj(frames=0)), out=None) == B.SNLS_OK


def test_the_binding_refuses_tensors_off_the_gpu():
    x = torch.zeros(2, 4)
    for f in (lambda: B.snls_norm(x), lambda: B.snls_norm_backward(x, x, x), lambda: B.snls_dropout(x, None, 0.0),
              lambda: B.snls_rotate(x, None, dict(B=1, T=1, C=4, H=1, W=2, HD=1, pairs=(1, 0, 0), theta=(9, 9, 9))),
              lambda: B.snls_rotate_points(x, None, dict(C=4)), lambda: B.snls_project_pack(x),
              lambda: B.snls_project(x, x, x)):
        with pytest.raises(ValueError):
            f()


# ------------------------------------------------------------- the plain forms --

def test_philox_known_answers():
    """The published test vectors of Philox 4x32-10."""
    assert R.philox([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 0xffffffff
    assert R.philox([f] * 4, [f] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    pi = [0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344]
    assert R.philox(pi, [0xa4093822, 0x299f31d0]) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_words_are_those_of_philox():
    seed, step, site = 0x0123456789abcdef - 2 ** 62, 2 ** 32 + 7, 5
    first = 2 ** 35 - 2
    got = R.words(first, 9, seed, step, site)
    for i, w in enumerate(got):
        e = first + i
        b = e >> 2
        s = seed & (2 ** 64 - 1)
        assert int(w) == R.philox([b & 0xffffffff, b >> 32, step & 0xffffffff, site], [s & 0xffffffff, s >> 32])[e & 3]


def test_dropout_keeps_its_share():
    keep = R.keep_mask((1 << 18,), (1234, 5), 0.25, 0).double()
    assert abs(float(keep.mean()) - 0.75) < 6 * math.sqrt(0.1875 / (1 << 18))  # six standard deviations


@pytest.mark.parametrize("shape", [(2, 5, 3, 4), (6, 7)])
def test_norm_gradient_formula(shape):
    g = torch.Generator().manual_seed(3)
    x, gy, gt = (torch.randn(shape, generator=g, dtype=torch.float64) for _ in range(3))
    C = R.rows(x).shape[-1]
    gamma, beta = (torch.randn(C, generator=g, dtype=torch.float64, requires_grad=True) for _ in range(2))
    x.requires_grad_(True)
    y, mean, rstd = R.norm(x, gamma, beta, 1e-5)
    ((y * gy).sum() + (x * gt).sum()).backward()
    (gx, gg, gb), _ = R.norm_backward(gy, x.detach(), torch.stack([mean, rstd]).detach(), gamma.detach(), gt)
    for a, b in ((gx, x.grad), (gg, gamma.grad), (gb, beta.grad)):
        assert float((a - b).abs().max()) < 1e-12 * (1 + float(b.abs().max()))
    # and against differences
    h = 1e-6
    for i in range(0, x.numel(), 7):
        f = []
        for s in (h, -h):
            z = x.detach().clone()
            z.view(-1)[i] += s
            f.append(float(((R.norm(z, gamma, beta, 1e-5)[0] * gy).sum() + (z * gt).sum()).detach()))
        assert abs((f[0] - f[1]) / (2 * h) - float(gx.reshape(-1)[i])) < 1e-7


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_depends_on_differences_and_inverts(interleaved):
    rp = dict(B=1, T=2, C=20, H=3, W=4, HD=2, pairs=(1, 2, 1), theta=(50.0, 10.0, 7.0), interleaved=interleaved)
    g = torch.Generator().manual_seed(5)
    q, k = (torch.randn(1, 2, 20, 3, 4, generator=g, dtype=torch.float64) for _ in range(2))
    times = torch.tensor([[3, 9]])
    dots = []
    for shift in (0, 1000):
        r = dict(rp, row0=shift, col0=-shift)
        a, b = R.rotate_video(q, times + shift, r), R.rotate_video(k, times + shift, r)
        dots.append(torch.einsum("bthcij,bshckl->bhtsijkl", a.view(1, 2, 2, 10, 3, 4), b.view(1, 2, 2, 10, 3, 4)))
    assert float((dots[0] - dots[1]).abs().max()) < 1e-11
    assert float((R.rotate_video(R.rotate_video(q, times, rp), times, rp, inverse=True) - q).abs().max()) < 1e-14
    pts = torch.tensor([[0, 2, 3], [0, 1, 0], [1, 0, 0]], dtype=torch.int32)
    tok = torch.stack([q[0, 1, :, 2, 3], q[0, 1, :, 1, 0], q[0, 1, :, 0, 0]])
    got = R.rotate_points(tok, pts, times[:, 1], rp)
    full = R.rotate_video(q, times, rp)
    assert torch.equal(got[0], full[0, 1, :, 2, 3]) and torch.equal(got[1], full[0, 1, :, 1, 0])
    assert float(got[2].abs().max()) == 0.0  # another video than there is


def test_quantised_codes_are_nearest_with_ties_to_even():
    s = np.float32(0.25)
    v = torch.tensor([[127 * 0.25, 0.125, 0.375, -0.625, 0.37, 0.0]], dtype=torch.float32)
    codes, scales = R.quantise(v)
    assert float(scales[0]) == float(s) and codes[0].tolist() == [127, 0, 2, -2, 1, 0]
    codes, scales = R.quantise(torch.tensor([[0.0, 0.0], [float("nan"), 1.0], [float("inf"), 1.0]]))
    assert codes.abs().max() == 0 and float(scales[0]) > 0 and bool(scales[1:].isnan().all())
