"""Workspaces that the caller brings: their bytes count, whatever their type."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from workloads import small_params

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


def _calls(p, dev):
    """(operation, call with a workspace) of every call that takes one."""
    g = torch.Generator(device=dev).manual_seed(3)
    q, k, v, go = (torch.randn(B.video_shape(p), device=dev, generator=g) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), device=dev, generator=g)
    d, i = B.snls_search(q, k, fl, p)
    bias = dict(radius=1, edges=[0.5, 2.0])
    gs = torch.randn(d.shape, device=dev, generator=g)
    w = d.softmax(-1)
    return [
        (B.SNLS_OP_AGGREGATE, lambda ws: B.snls_aggregate(v, d, i, p, 0.2, workspace=ws)),
        (B.SNLS_OP_AGGREGATE_STACKED, lambda ws: B.snls_aggregate_stacked(v, d, i, p, 0.2, workspace=ws)),
        (B.SNLS_OP_BIAS_BACKWARD, lambda ws: B.snls_bias_backward(gs, d, i, p, bias, workspace=ws)),
        (B.SNLS_OP_BACKWARD, lambda ws: B.snls_backward(q, k, v, fl, d, i, go, p, 0.2, workspace=ws)[2]),
        (B.SNLS_OP_BACKWARD, lambda ws: B.snls_backward_scores(q, k, v, fl, d, i, go, p, 0.2, workspace=ws)[4]),
        (B.SNLS_OP_GATHER_STACKED, lambda ws: B.snls_gather_stacked(v, w, i, p, workspace=ws)),
    ]


def test_bytes_count(dev):
    p = small_params(T=2, C=8, H=20, W=21, ps=1, k=4)
    for op, call in _calls(p, dev):
        need = B.snls_workspace_size(op, p)
        if need == 0:
            continue
        want = call(None)
        for t in (torch.uint8, torch.float16, torch.float64):
            size = torch.empty((), dtype=t).element_size()
            got = call(torch.empty(-(-need // size), dtype=t, device=dev))
            assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())
        # a quarter of the bytes is refused, though its bytes are as many as the floats asked for
        with pytest.raises(B.SnlsError):
            call(torch.empty(need - 1, dtype=torch.uint8, device=dev))
        with pytest.raises(B.SnlsError):
            call(torch.empty((need + 3) // 4, dtype=torch.uint8, device=dev))
        for bad in (torch.empty(1, device=dev).expand(need), torch.empty(need // 2, 4, device=dev)[:, 1:],
                    torch.empty(need)):
            with pytest.raises(ValueError):
                call(bad)
