"""The choice of experts reads a logit as it is: infinite logits and prices, the largest finite ones beside them, ties
among them, NaN. Expected by hand and by the oracle; all row lengths of the kernel, both ways of planning."""

import math

import numpy as np
import pytest

from oracle import moe_oracle as mo

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def mm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_07971_gb300 import build, moe
    build.build()
    m = moe.Moe()
    yield m
    m.synchronize()
    m.close()


def test_by_hand(mm):
    inf, nan, big = math.inf, math.nan, torch.finfo(torch.float32).max
    z = torch.tensor([[big, inf, 0.0], [inf, inf, big], [nan, -inf, 1.0], [inf, nan, inf]], device="cuda")
    assert mm.route(z, 3).idx.tolist() == [[1, 0, 2], [0, 1, 2], [2, -1, -1], [0, 2, -1]]
    # inf - 1e38 is inf; big - 1e38 is not
    p = torch.tensor([1e38, 0.0, 0.0], device="cuda")
    assert mm.route(z, 3, prices=p).idx.tolist() == [[1, 0, 2], [0, 1, 2], [2, -1, -1], [0, 2, -1]]
    # an infinite price closes; inf - inf is no number
    p = torch.tensor([inf, 0.0, 0.0], device="cuda")
    assert mm.route(z, 3, prices=p).idx.tolist() == [[1, 2, -1], [1, 2, -1], [2, -1, -1], [2, -1, -1]]
    # a price of -inf makes every finite logit's profit infinite, equal among them; -inf + inf is no number
    p = torch.tensor([-inf, -inf, 0.0], device="cuda")
    assert mm.route(z, 3, prices=p).idx.tolist() == [[0, 1, 2], [0, 1, 2], [2, -1, -1], [0, 2, -1]]
    p = torch.tensor([nan, 0.0, nan], device="cuda")
    assert mm.route(z, 3, prices=p).idx.tolist() == [[1, -1, -1], [1, -1, -1], [-1, -1, -1], [-1, -1, -1]]


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("E", [7, 40, 100, 250, 500, 1000])
@pytest.mark.parametrize("T", [9, 300])
def test_extremes_against_the_oracle(mm, T, E, dt):
    rng = np.random.default_rng(T * E)
    top = torch.finfo(DT[dt]).max
    pool = torch.tensor([math.inf, -math.inf, math.nan, top, -top, 0.0, -0.0, 1.0, -2.5], device="cuda").to(DT[dt])
    z = pool[torch.as_tensor(rng.integers(0, 9, (T, E))).cuda()]
    z[::3] = torch.as_tensor(rng.normal(size=(len(range(0, T, 3)), E))).cuda().to(DT[dt])
    extreme = np.array([math.inf, -math.inf, math.nan, 3.4028234663852886e38, 1e38, 0.0, -0.0, 1.0, -2.5], np.float32)
    for prices in (None, np.zeros(E, np.float32), extreme[rng.integers(0, 9, E)],
                   np.maximum(0, rng.normal(size=E)).astype(np.float32)):
        k = min(5, E)
        r = mm.route(z, k, prices=None if prices is None else torch.as_tensor(prices).cuda())
        want = mo.choose(z.float().cpu().numpy(), k, prices)
        assert np.array_equal(r.idx.cpu().numpy(), want)
        counts, offsets, rows, pos = mo.plan(want, E)
        for got, w in ((r.counts, counts), (r.offsets, offsets), (r.rows, rows), (r.pos, pos)):
            assert np.array_equal(got.cpu().numpy(), w)
