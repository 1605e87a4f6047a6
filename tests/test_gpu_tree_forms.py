"""Tree attention's forms for large batches, and calls whose device arrays do not fit the host's plan, against the
definitions in 64 bits (tests/tree_reference.py) and against themselves bit for bit."""
import numpy as np
import pytest
import torch

from paper_2608_22167_amd import mcpu
from tests import tree_reference as R
from tests.test_gpu_tree import LAYOUTS, PAGE, Case, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# ------------------------------------------------------------------------------ a sink of -inf


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[3], LAYOUTS[6]], ids=str)
@pytest.mark.parametrize("lengths", [(100, 5), (2900, 40)], ids=["one_split", "splits"])
def test_a_sink_of_minus_infinity_is_no_sink(layout, lengths):
    """Beside keys it adds nothing to the normaliser; without a key (all pages missing) it gives zeros as no sink does."""
    sinks = torch.from_numpy(np.resize([float("-inf"), 0.5], layout[0]).astype(np.float32))
    c = Case(layout, lengths, trees(np.random.default_rng(60), [9, 4]), 0, 61, sinks=sinks)
    c.check()
    for b in range(2):
        d = Case(layout, lengths, trees(np.random.default_rng(60), [9, 4]), 0, 61, sinks=sinks)
        d.table[b] = -1
        got = d.check(errors=mcpu.DEVERR_PAGE)
        assert (got[d.cu[b]:d.cu[b + 1]] == 0).all()
