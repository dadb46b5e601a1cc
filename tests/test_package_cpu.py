"""What the package offers at its top: every call of the position bias and of
the frame cache, with what sizes their buffers."""
import paper_2309_16849_amd as pkg
from paper_2309_16849_amd import snls as B


def test_buffers_of_the_operators_can_be_sized_from_the_package():
    bias, cp = dict(radius=2, edges=[0.5, 2.0]), dict(B=1, slots=3, C=40, H=17, W=20, HD=2, block=8)
    assert pkg.bias_table_shape(bias, 4) == (4, 5, 5, 5)
    assert pkg.cache_shapes(cp) == ((1, 3, 2, 17, 20, 32), (1, 3, 2, 3, 3))
    p = dict(B=1, T=2, C=4, H=8, W=8, HD=1, ws=3, wt=1, ps=1, stride0=1, stride1=1.0, k=3, dist_type=0)
    assert pkg.snls_workspace_size(pkg.SNLS_OP_BIAS_BACKWARD, p) > 0
    for name in B.SYMBOLS:
        if name.startswith(("snls_bias", "snls_cache", "snls_backward")):
            assert getattr(pkg, name) is getattr(B, name)
