"""Log probabilities of rows with NaN: the largest classes are those of the
other scores, with NaN for their log probabilities; places beyond them hold -1
and -inf, as places beyond the scores that are not -inf do."""
import math

import pytest
import torch

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("top", [4, 7, 17])
@pytest.mark.parametrize("v", [5, 19, 300, 3000, 40_000, 300_000])
def test_classes_of_a_row_with_nan(v, top, ty):
    x = torch.full((3, v), -math.inf)
    x[:, 1], x[:, v - 2], x[:, v // 2] = 2.0, 3.0, -1.0
    x[1, 0] = math.nan
    x[1, v - 1] = math.nan
    ids = torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda")
    logp, lse, ent, ti, tp = ezsp.log_probs(x.to("cuda", ty), ids, top, True)
    want = [v - 2, 1, v // 2] + [-1] * (top - 3)
    assert ti.tolist() == [want] * 3
    assert bool((tp[:, 3:] == -math.inf).all())
    assert bool(tp[1, :3].isnan().all())
    assert bool(tp[[0, 2], :3].isfinite().all())
    for t in (logp, lse, ent):
        assert bool(t[1].isnan()) and not bool(t[[0, 2]].isnan().any())
    assert float(logp[2]) == -math.inf


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("v", [5, 300, 40_000])
def test_a_row_of_nan_alone(v, ty):
    x = torch.zeros((3, v), dtype=ty, device="cuda")
    x[1] = math.nan
    logp, lse, ent, ti, tp = ezsp.log_probs(
        x, torch.zeros(3, dtype=torch.int32, device="cuda"), 2, True)
    assert ti.tolist() == [[0, 1], [-1, -1], [0, 1]]
    assert bool((tp[1] == -math.inf).all())
    assert bool(lse[1].isnan()) and bool(ent[1].isnan()) and \
        bool(logp[1].isnan())
