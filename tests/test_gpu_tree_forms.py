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


# ------------------------------------------------------------------------------ the forms of large batches

# Over 12288 (page, KV head) pairs in contexts of more than 24 pages, also inside the window of 2300: by the columns of
# the largest tree (nodes times query heads per KV head) the streaming form (up to 32), two column tiles a wavefront in
# workgroups of two (up to 128) or of four (above).
BIG = [((32, 32, 64, "bf16"), 9), ((64, 32, 64, "bf16"), 20), ((64, 32, 64, "bf16"), 64), ((128, 32, 64, "bf16"), 40)]
WINDOW = 2300
big = pytest.mark.parametrize("layout,n", BIG, ids=str)


def big_case(layout, n, window, seed=70, **kw):
    rng = np.random.default_rng(seed)
    return Case(layout, [2500, 2481, 2490], trees(rng, [n, n - 1, n - 2]), window, seed + 1, **kw)


@big
@pytest.mark.parametrize("window", [0, WINDOW])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_contents_that_no_node_sees_in_large_batches(layout, n, window, bad):
    """NaN and infinities behind the trees, in free pages and left of every window change no bit; one value at the
    window's left end reaches the roots alone, and one node's K and V reach the nodes of its branch."""
    c = big_case(layout, n, window)
    clean = c.run()
    assert torch.isfinite(clean.float()).all()
    ko, vo = R.slot_offsets(64)

    def put(b, slot, what=(0, 1)):
        for i, (x, off) in enumerate(((c.k, ko), (c.v, vo))):
            if i in what:
                x[int(c.table[b, slot // PAGE])][:, torch.from_numpy(off[slot % PAGE])] = bad

    free = np.setdiff1d(np.arange(c.n_pages), c.table)
    c.k[torch.from_numpy(free)] = bad
    c.v[torch.from_numpy(free)] = bad
    for b in range(3):
        end = int(c.seq[b] + c.cu[b + 1] - c.cu[b])
        for slot in range(end, -(-end // PAGE) * PAGE):
            put(b, slot)
        if window:
            lo = int(c.seq[b]) - window + 1
            for slot in range(lo // PAGE * PAGE, lo):
                put(b, slot)
    assert same(c.run(), clean)
    hit = np.zeros(c.T, bool)
    for b, node in ((0, 2), (2, n - 4)):
        par = c.par[c.cu[b]:c.cu[b + 1]]
        put(b, int(c.seq[b]) + node, (0, 1) if b else (1,))
        hit[c.cu[b]:c.cu[b + 1]] |= R.visible(par, 0, 0)[:, node]
    if window:  # a value: only nodes at depth 0 reach that far
        put(1, int(c.seq[1]) - window + 1, (1,))
        hit[c.cu[1]:c.cu[2]] |= R.depths(c.par[c.cu[1]:c.cu[2]]) == 0
    got = c.run()
    assert same(got[~hit], clean[~hit])
    assert not torch.isfinite(got[hit].float()).any()


@big
@pytest.mark.parametrize("window", [0, WINDOW])
def test_missing_pages_in_large_batches(layout, n, window):
    """Single pages of either half of a step, a run of them, the window's first and a tree's own last page."""
    c = big_case(layout, n, window, 72, sinks=None)
    first = max(0, 2481 - window + 1) // PAGE if window else 0
    for b, lp in ((0, 40), (0, 77), (0, 110), (1, first), (1, 60), (1, 61), (1, 62), (1, 63), (2, (2490 + n - 3) // PAGE)):
        c.table[b, lp] = -1 if lp % 2 else c.n_pages + b
    c.check(errors=mcpu.DEVERR_PAGE)


@big
def test_values_that_are_not_finite_beside_missing_pages(layout, n):
    """Pages beside a missing one take the step with masked keys: infinite values on them reach every node, and only
    that sequence's."""
    c = big_case(layout, n, 0, 73)
    for lp in (41, 90):
        c.table[1, lp] = -1
    clean = c.run(errors=mcpu.DEVERR_PAGE)
    c.v[int(c.table[1, 40])] = float("inf")
    c.v[int(c.table[1, 91])] = float("inf")
    got = c.run(errors=mcpu.DEVERR_PAGE)
    mine = slice(int(c.cu[1]), int(c.cu[2]))
    assert (got[mine].float() == float("inf")).all()
    got[mine] = clean[mine]
    assert same(got, clean)


@big
@pytest.mark.parametrize("window", [0, WINDOW])
def test_large_scores_in_large_batches(layout, n, window):
    """Scores of hundreds, so that the maximum is raised again and again in either column tile; sinks of +-30."""
    sinks = torch.from_numpy(np.resize([30.0, -30.0, 0.5, 4.0], layout[0]).astype(np.float32))
    big_case(layout, n, window, 74, q_scale=50.0, sinks=sinks).check()


@big
@pytest.mark.parametrize("window", [0, WINDOW])
def test_rising_scores_in_large_batches(layout, n, window):
    """Keys that grow along the context: every step raises some column's maximum."""
    c = big_case(layout, n, window, 75)
    ko, _ = R.slot_offsets(64)
    for b in range(3):
        for lp in range(c.table.shape[1]):
            if c.table[b, lp] >= 0:
                c.k[int(c.table[b, lp])] *= 1 + lp / 8
    c.check()


@big
@pytest.mark.parametrize("window", [0, WINDOW])
def test_large_batches_repeat_their_bits_anywhere(layout, n, window):
    """From run to run, with other pages, on a used workspace, and for a branch among other branches."""
    c = big_case(layout, n, window, 76)
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(c.shape, 3, c.T))
    a = c.run(ws=ws)
    for _ in range(3):
        assert same(a, c.run(ws=ws))
    perm = np.random.default_rng(77).permutation(c.n_pages)
    inv = np.argsort(perm)
    c.k, c.v = c.k[torch.from_numpy(perm)], c.v[torch.from_numpy(perm)]
    c.table = np.where(c.table >= 0, inv[np.maximum(c.table, 0)], -1).astype(np.int32)
    assert same(a, c.run(ws=ws))


@pytest.mark.parametrize("window", [1, 3, 6])
def test_window_shorter_than_the_branch_in_the_streaming_form(window):
    """Many short windows: over 12288 (page, KV head) pairs without a split."""
    rng = np.random.default_rng(78)
    seq = rng.integers(30, 90, 290)
    tr = [[i - 1 for i in range(8)] if b % 2 else R.random_tree(rng, 8, 3) for b in range(290)]
    Case((32, 32, 64, "bf16"), seq, tr, window, 79).check()


@pytest.mark.parametrize("n", [4, 12, 20])
def test_large_batches_of_more_than_256_sequences(n):
    """The same three forms from the plan's records: many short contexts and some in splits."""
    rng = np.random.default_rng(80 + n)
    seq, sizes = rng.integers(0, 40, 280), rng.integers(0, 3, 280)
    seq[::7], sizes[::7] = rng.integers(500, 900, 40), rng.integers(1, n + 1, 40)
    sizes[7] = n
    Case(LAYOUTS[2], seq, trees(rng, sizes), 0, 81).check()
