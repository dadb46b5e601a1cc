"""Memory that the binding allocates for a call on another stream than the
current one is not given to other work before the call is done."""
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
    g = torch.Generator(device=dev).manual_seed(3)
    q, k, v, go = (torch.randn(B.video_shape(p), device=dev, generator=g) for _ in range(4))
    fl = torch.randn(B.flow_shape(p), device=dev, generator=g)
    d, i = B.snls_search(q, k, fl, p)
    bias = dict(radius=1, edges=[0.5, 2.0])
    table = torch.randn(B.bias_table_shape(bias, p["HD"]), device=dev, generator=g)
    gs = torch.randn(d.shape, device=dev, generator=g)
    cp = dict(B=1, slots=2, C=p["C"], H=p["H"], W=p["W"], HD=p["HD"], block=8)
    cache = B.cache_alloc(cp, dev)
    for s in range(2):
        B.snls_cache_store(k[:, s].contiguous(), v[:, s].contiguous(), torch.full((1,), s, dtype=torch.int32, device=dev),
                           cp, cache)
    ages = torch.ones(1, 2, dtype=torch.int32, device=dev)
    frame, pts = q[:, 0].contiguous(), torch.zeros(50, 3, dtype=torch.int32, device=dev)
    tok = torch.randn(50, p["C"], device=dev, generator=g)
    return {
        "search": lambda **kw: B.snls_search(q, k, fl, p, **kw), "aggregate": lambda **kw: B.snls_aggregate(v, d, i, p, **kw),
        "stacked": lambda **kw: B.snls_aggregate_stacked(v, d, i, p, **kw),
        "backward": lambda **kw: B.snls_backward(q, k, v, fl, d, i, go, p, **kw)[2:3],
        "scores": lambda **kw: B.snls_backward_scores(q, k, v, fl, d, i, go, p, **kw)[4:],
        "bias": lambda **kw: B.snls_bias(d, i, table, p, bias, **kw),
        "table": lambda **kw: B.snls_bias_backward(gs, d, i, p, bias, **kw),
        "attend": lambda **kw: B.snls_cache_attend(frame, None, ages, cache, cp, 3, **kw),
        "points": lambda **kw: B.snls_cache_attend_points(tok, pts, None, ages, cache, cp, 3, **kw),
    }


@pytest.mark.parametrize("name", ["search", "aggregate", "stacked", "backward", "scores", "bias", "table", "attend",
                                  "points"])
def test_memory_of_a_call_on_another_stream(dev, name, monkeypatch):
    p = small_params(T=2, C=8, H=40, W=41, ps=1, k=4)
    call = _calls(p, dev)[name]
    flat = lambda x: list(x) if isinstance(x, (tuple, list)) else [x]  # noqa: E731
    want = [x.clone() for x in flat(call())]
    spaces, make = [], B.workspace_for

    def noted(*a, **kw):
        spaces.append(make(*a, **kw))
        return spaces[-1]

    monkeypatch.setattr(B, "workspace_for", noted)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)  # some 10 ms of a counting kernel
        outs = flat(call(stream=side))
        held = [(t.data_ptr(), t.numel()) for t in outs + spaces]
        shapes = [t.shape for t in outs]
        del outs
        spaces.clear()
        fresh = [torch.full((n,), float("nan"), device=dev) for _, n in held]  # other work of the current stream
        assert not side.query()
        assert not {t.data_ptr() for t in fresh} & {at for at, _ in held}
        torch.cuda.synchronize()
        del fresh
    outs = flat(call(stream=side))
    torch.cuda.synchronize()
    for a, b, s in zip(outs, want, shapes):
        assert a.shape == s and float((a - b).abs().max()) <= 1e-5 * float(b.abs().max())
