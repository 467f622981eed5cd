"""The linear layer's cross-entropy at sizes that between them run every tile kind in every part of the
work (test_linear_ce_kinds.py says so), against the formulas in 64 bits.  Tolerances: test_gpu_linear_ce.py's."""
import math

import pytest

torch = pytest.importorskip("torch")

import linear_ce_kinds as kinds  # noqa: E402
from paper_2609_10018_amd import ffi  # noqa: E402
from test_gpu_linear_ce import BF, F32, Case, holds  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ffi.load_library()


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("es,rows,dim,classes", kinds.CASES)
def test_every_kind(es, rows, dim, classes, weights):
    """Rows that do not count, by their labels or their weights, hold NaN: what is summed over rows must
    leave them out by their bits or have set them aside."""
    case = Case(BF if es == 2 else F32, rows, dim, classes, bias=weights, weights=weights, pad=8 if weights else 0)
    case.y[3::7] = -1
    left_out = case.y < 0 if case.rw is None else (case.y < 0) | (case.rw == 0)
    counts = ~left_out
    ref = case.reference()
    case.x[left_out] = math.nan
    loss, lse = case.forward()
    none = left_out if case.rw is None else case.rw == 0
    for n, t in (("loss", loss), ("lse", lse)):
        holds(n, t[counts], tuple(v[counts] for v in ref[n]))
        assert (t[none] == 0).all() if weights else t[none].isnan().all()
    got = case.backward(lse)
    for n, t in got.items():
        holds(n, t, ref[n])
    assert (got["dx"][left_out] == 0).all()
    again = case.backward(lse)
    assert all(torch.equal(got[n], again[n]) for n in got)
