"""Attention over cached frames where NaN values lie behind weights that
vanish: a table entry that masks a frame step (the type's lowest value or
-1e4, both finite logits) leaves its candidates a weight of 0 in fp32, and
values of weight 0 are not read (include/snls.h) -- whatever the order of the
slots and however they are split over waves.  Tolerances as in
test_gpu_frame_cache.py."""
import pytest
import torch

from paper_2309_16849_amd import snls as B
from tests import attention64 as R
from tests.test_gpu_frame_cache import _both, _cp, _filled, _points, _tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    return torch.device("cuda:0")


FORMS = [  # channels, heads, window, slots, frame: few waves (slots split over four), many (not split)
    (16, 1, 5, 5, (20, 21)), (64, 1, 7, 5, (20, 21)), (96, 1, 5, 6, (18, 17)), (160, 1, 4, 5, (14, 15)),
    (256, 1, 5, 5, (12, 13)), (64, 4, 5, 3, (130, 130)), (128, 2, 7, 2, (190, 180)),
]


@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, -1e4], ids=["lowest", "-1e4"])
@pytest.mark.parametrize("masked", [(0,), (-1,), (0, 1), (1,)], ids=str)
@pytest.mark.parametrize("C,HD,ws,slots,frame", FORMS, ids=str)
def test_nan_behind_a_mask(dev, C, HD, ws, slots, frame, masked, low):
    masked = [s % slots for s in masked][:slots - 1]  # one slot at least is left
    cp = _cp(C=C, HD=HD, H=frame[0], W=frame[1], slots=slots)
    g = torch.Generator().manual_seed(7)
    cache, _, _ = _filled(cp, dev)
    for s in masked:
        cache[2].view(torch.uint8)[0, s] = 0x7F  # NaN
    bias = dict(radius=2, edges=[1.0])
    table = torch.randn(B.bias_table_shape(bias, HD), generator=g)
    table[:, 0] = low  # frame step -2
    ages = torch.ones(1, slots, dtype=torch.int32)
    ages[0, masked] = 2
    q = torch.randn(1, C, *frame, generator=g)
    # inside the frame: every query has candidates that are not masked
    fl = torch.rand(1, slots, 2, *frame, generator=g) - 0.5
    print("masked", cp, ws, masked, flush=True)
    a, b, qa, allp, fa = _both(dev, cp, ws, q, fl, ages, cache, 0.5, table, bias)
    assert bool(a.isfinite().all()) and bool(b.isfinite().all())
    pick = torch.randint(0, qa.shape[0], (30,), generator=g)
    to = lambda x: x.to(dev)  # noqa: E731
    few = B.snls_cache_attend_points(to(qa[pick]), to(allp[pick]), to(fa[pick]), to(ages), cache, cp, ws, 0.5,
                                     table=to(table), bias=bias).cpu()
    live = [s for s in range(slots) if s not in masked]
    kv, vv = (R.decoded(cache[i][:, live].contiguous(), cache[i + 1][:, live].cpu(), dict(cp, slots=len(live)))
              for i in (0, 2))
    ref, big = R.attend(qa[pick], allp[pick], fa[pick][:, live], ages[:, live], kv, vv, dict(cp, slots=len(live)), ws,
                        0.5, table, bias)
    tol = _tol(qa[pick], kv, vv, cp, ws, 0.5, big, table[:, 1:])
    for o in (a[pick], b[pick], few):
        assert float((o.double() - ref).abs().max()) <= tol


def test_all_masked_keeps_the_softmax(dev):
    """Where every candidate is masked alike, the softmax is that of what is left beside the mask: NaN shows."""
    cp = _cp(C=16, HD=1, H=9, W=10, slots=2)
    cache, _, _ = _filled(cp, dev)
    cache[2].view(torch.uint8)[0, 0] = 0x7F
    bias = dict(radius=0, edges=[])
    table = torch.full((1, 1, 1, 1), torch.finfo(torch.float32).min)
    q = torch.zeros(1, 16, 9, 10)
    for o in _both(dev, cp, 3, q, None, torch.zeros(1, 2, dtype=torch.int32), cache, 1.0, table, bias)[:2]:
        assert bool(o.isnan().all())
