"""Numbers that a C field does not hold are refused, not taken modulo its size."""
import pytest
import torch

from paper_2309_16849_amd import snls as B

ROT = dict(B=1, T=2, C=16, H=5, W=6, HD=2, pairs=(1, 2, 1), theta=(100.0, 100.0, 100.0))


@pytest.mark.parametrize("key", ["B", "T", "C", "H", "W", "HD", "interleaved", "row0", "col0"])
@pytest.mark.parametrize("more", [2 ** 32, 2 ** 31, -2 ** 31 - 1, 2 ** 64])
def test_rotary_numbers_past_32_bits(key, more):
    with pytest.raises(ValueError):
        B.rotate_from_dict(dict(ROT, **{key: ROT.get(key, 0) + more if more > 0 else more}))


@pytest.mark.parametrize("axis", range(3))
def test_rotary_pairs_past_32_bits(axis):
    pairs = list(ROT["pairs"])
    pairs[axis] += 2 ** 32
    with pytest.raises(ValueError):
        B.rotate_from_dict(dict(ROT, pairs=pairs))


def test_rotary_numbers_of_32_bits_are_kept():
    prm = B.rotate_from_dict(dict(ROT, row0=-2 ** 31, col0=2 ** 31 - 1))
    assert (prm.row0, prm.col0) == (-2 ** 31, 2 ** 31 - 1)


@pytest.mark.parametrize("site", [-1, 2 ** 32, 2 ** 40 + 5])
def test_sites_past_32_bits(site):
    """Two sites must not share a mask."""
    with pytest.raises(ValueError):
        B.norm_params(8, 3, 20, 1e-5, 0.5, site)
    with pytest.raises(ValueError):
        B.dropout_site(site)


def test_sites_of_32_bits_are_kept():
    assert B.norm_params(8, 3, 20, 1e-5, 0.5, 2 ** 32 - 1).site == B.dropout_site(2 ** 32 - 1) == 2 ** 32 - 1


def test_channels_past_32_bits_stay_too_many():
    """2^32 + 8 channels are not 8: the library refuses them."""
    lib, many = B.load_library(), 2 ** 32 + 8
    prm = B.norm_params(many, 1, 1, 1e-5, 0.0, 0)
    assert lib.snls_norm(*[0x1000] * 5, prm, *[0x1000] * 3, None) == B.SNLS_ERR_UNSUPPORTED
    for prm in (B.project_params(many, 4, 1, 1, 1), B.project_params(4, many, 1, 1, 1)):
        assert lib.snls_project(*[0x1000] * 4, prm, 0x1000, None) == B.SNLS_ERR_UNSUPPORTED
        assert lib.snls_project_pack(0x1000, prm, 0x1000, 0x1000, None) == B.SNLS_ERR_UNSUPPORTED


def test_theta_past_fp32():
    with pytest.raises(ValueError):
        B.rotate_from_dict(dict(ROT, theta=(1e39, 1.0, 1.0)))
    assert [float(t) for t in B.rotate_from_dict(dict(ROT, theta=(1e4, 0.1, 3e38))).theta] == [
        1e4, float(torch.tensor(0.1)), float(torch.tensor(3e38))]
