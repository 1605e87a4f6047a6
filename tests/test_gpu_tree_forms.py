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


# ------------------------------------------------------------------------------ trees that the plan has no place for


def _left_out(c, ws, clean, rows, errors=mcpu.DEVERR_PLAN, **device):
    """The call with other arrays on the device: the given rows of o stay as they were, all others have their bits."""
    got = c.run(errors=errors, ws=ws, device=device)
    out = np.zeros(c.T, bool)
    out[rows] = True
    assert (got[out] == 7).all(), "rows of a tree that is left out were written"
    assert same(got[~out], clean[~out])


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[3]], ids=str)
def test_trees_left_out_of_splits_keep_their_rows(layout):
    """Over the records and partial rows that a complete call left in the workspace."""
    c = Case(layout, [900, 40, 1500], trees(np.random.default_rng(62), [20, 8, 5]), 0, 63)
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(c.shape, 3, c.T))
    clean = c.run(ws=ws)
    seq = lambda *a: dict(seq=list(a))  # noqa: E731
    first, last = np.arange(20), np.arange(28, 33)
    _left_out(c, ws, clean, first, **seq(-5, 40, 1500))
    _left_out(c, ws, clean, last, **seq(900, 40, 1 << 30))
    _left_out(c, ws, clean, np.arange(28), **seq(-1, -1, 1500))
    # rows that no tree covers
    _left_out(c, ws, clean, np.arange(20), cu=[20, 20, 28, 33])
    _left_out(c, ws, clean, last, cu=[0, 20, 28, 28])
    _left_out(c, ws, clean, np.arange(33), cu=[0, -3, -9, 28])
    assert same(c.run(ws=ws), clean)


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[3]], ids=str)
def test_trees_whose_splits_pass_the_plan_are_left_out(layout):
    """A context that is longer on the device takes the places of the trees behind it: what has no place for all of its
    splits is left out, and what has one is right."""
    c = Case(layout, [900, 1500, 900], trees(np.random.default_rng(64), [7, 6, 5]), 0, 65)
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(c.shape, 3, c.T))
    clean = c.run(ws=ws)
    # tree 0 as short as one split frees places that nobody takes; the others are where they were
    got = c.run(errors=mcpu.DEVERR_PLAN, ws=ws, device=dict(seq=[100, 1500, 900]))
    assert same(got[7:], clean[7:]) and not (got[:7] == 7).any()
    # tree 0 as long as tree 1 needs more: the last tree's splits pass the end
    c.table[0, :c.table.shape[1] - 2] = c.table[1, :c.table.shape[1] - 2]
    clean = c.run(ws=ws)
    got = c.run(errors=mcpu.DEVERR_PLAN, ws=ws, device=dict(seq=[1480, 1500, 900]))
    assert same(got[7:13], clean[7:13]) and (got[13:] == 7).all()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[3]], ids=str)
def test_trees_left_out_of_more_than_256_sequences(layout):
    rng = np.random.default_rng(66)
    seq, sizes = rng.integers(0, 60, 301), rng.integers(1, 5, 301)
    seq[[7, 200, 300]] = 3000
    c = Case(layout, seq, trees(rng, sizes), 0, 67)
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(c.shape, 301, c.T))
    clean = c.run(ws=ws)
    rows = lambda *b: np.concatenate([np.arange(c.cu[i], c.cu[i + 1]) for i in b])  # noqa: E731
    for out in ([7], [200, 300], [0, 7, 8, 299], [300]):
        dev = c.seq.copy()
        dev[out] = -1
        _left_out(c, ws, clean, rows(*out), seq=dev)
    cu = c.cu.copy()
    cu[301] = cu[300]
    _left_out(c, ws, clean, rows(300), cu=cu)
    assert same(c.run(ws=ws), clean)
