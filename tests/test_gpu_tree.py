"""Trees of drafted tokens on the GPU against the definitions in 64 bits
(tests/tree_reference.py): attention over layouts, lengths, windows, splits and
contents that no node sees; acceptance; commit; and a step of all of them. The
tolerances are the error bounds derived there."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2608_22167_amd import mcpu, workload as W
from tests import tree_reference as R

pytestmark = pytest.mark.gpu

PAGE = 16
# query heads, KV heads, head dim, dtype
LAYOUTS = [(8, 2, 32, "f32"), (4, 1, 64, "f32"), (64, 8, 64, "bf16"), (8, 2, 64, "bf16"), (16, 1, 32, "bf16"),
           (32, 2, 64, "bf16"), (6, 6, 64, "bf16")]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


def shape_of(layout, window=0):
    hq, hkv, d, t = layout
    return replace(W.TINY if t == "f32" else W.GPT_OSS_20B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, window=window)


class Case:
    """Sequences with trees in a pool of random values, on the host and the GPU."""

    def __init__(self, layout, seq_lens, trees, window=0, seed=0, q_scale=1.5, n_pages=None, sinks="normal"):
        rng = np.random.default_rng(seed)
        self.shape = s = shape_of(layout, window)
        self.window, self.bf16 = window, s.dtype == "bf16"
        self.seq = np.array(seq_lens, np.int32)
        n = np.array([len(t) for t in trees])
        self.cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.par = np.array([p for t in trees for p in t], np.int32)
        first = (np.maximum(0, self.seq - window + 1) if window else 0 * self.seq) // PAGE
        last = np.maximum((self.seq + n + PAGE - 1) // PAGE, first)
        need = int((last - first).sum())
        self.n_pages = n_pages or need + 3
        perm = rng.permutation(self.n_pages)[:need]
        self.table = np.full((len(seq_lens), max(1, int(last.max()) + 1)), -1, np.int32)
        at = 0
        for b in range(len(seq_lens)):
            self.table[b, first[b]:last[b]] = perm[at:at + last[b] - first[b]]
            at += last[b] - first[b]
        self.T, t = int(self.cu[-1]), s.torch_dtype
        block = (self.n_pages, s.n_kv_heads, PAGE * s.head_dim)
        draw = lambda *shp: torch.from_numpy(rng.standard_normal(shp).astype(np.float32))  # noqa: E731
        self.k, self.v = draw(*block).to(t), draw(*block).to(t)
        self.q = (draw(self.T, s.n_q_heads, s.head_dim) * q_scale).to(t)
        self.sinks = draw(s.n_q_heads) if isinstance(sinks, str) else sinks

    def reference(self):
        d = lambda x: x.double().numpy()  # noqa: E731
        return R.attention(d(self.q), d(self.k), d(self.v), self.table, self.seq, self.cu, self.par,
                           None if self.sinks is None else self.sinks.numpy(), self.window, self.bf16)

    def run(self, errors=0, device=None, guard=2, ws=None, stream=None):
        """tree_attention with `guard` rows around o that have to stay as they were."""
        s = self.shape
        page = (self.n_pages, s.n_kv_heads, PAGE, s.head_dim)
        k, v = self.k.cuda().view(page), self.v.cuda().view(page)
        pool = mcpu.KVPool(s, k, v)
        o = torch.full((self.T + 2 * guard, s.n_q_heads * s.head_dim), 7.0, dtype=s.torch_dtype, device="cuda")
        ws = mcpu.workspace(mcpu.tree_attention_workspace_size(s, len(self.seq), self.T)) if ws is None else ws
        dev = dict(table=self.table, seq=self.seq, cu=self.cu, par=self.par, **{})
        dev.update(device or {})
        up = {k_: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda() for k_, a in dev.items()}
        q = self.q.cuda()
        sinks = None if self.sinks is None else self.sinks.cuda()
        torch.cuda.synchronize()
        mcpu.tree_attention(s, sinks, pool, up["table"], up["seq"], up["cu"], up["par"], self.seq, self.cu, q,
                            o[guard:guard + self.T], ws, stream)
        torch.cuda.synchronize()
        assert mcpu.mcpu_check_device_errors(ws) == errors
        assert (o[:guard] == 7).all() and (o[guard + self.T:] == 7).all(), "rows outside the trees were written"
        assert torch.equal(k.cpu().view(self.k.shape).view(torch.uint8), self.k.view(torch.uint8))
        return o[guard:guard + self.T].cpu().view(self.T, s.n_q_heads, s.head_dim)

    def check(self, **kw):
        got = self.run(**kw).double().numpy()
        ref, tol = self.reference()
        assert np.isfinite(got).all()
        off = np.abs(got - ref) / tol
        print(f"  worst error {off.max():.3f} of its bound")
        assert off.max() <= 1, (off.max(), np.unravel_index(off.argmax(), off.shape))
        return got


def trees(rng, sizes, reach=4):
    return [R.random_tree(rng, n, reach) for n in sizes]


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("window", [0, 128])
def test_attention_layouts_and_lengths(layout, window):
    """Empty and one-token contexts, page borders, trees of 0, 1 and 64 nodes."""
    rng = np.random.default_rng(1)
    Case(layout, [0, 1, 15, 16, 17, 0, 200, 700, 31], trees(rng, [1, 64, 0, 5, 16, 33, 2, 64, 17]), window, 2).check()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[5]], ids=str)
@pytest.mark.parametrize("window", [1, 3, 20, 33])
def test_attention_window_shorter_than_the_branch(layout, window):
    chain = [i - 1 for i in range(64)]
    rng = np.random.default_rng(3)
    Case(layout, [100, 5, 0, 47], [chain, chain[:40], chain, R.random_tree(rng, 50, 2)], window, 4).check()


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("n", [1, 3, 16, 64])
def test_attention_of_one_long_context_in_splits(layout, n):
    """Several splits of one context, joined by the combine."""
    Case(layout, [3001], trees(np.random.default_rng(n), [n]), 0, 5 + n).check()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[3]], ids=str)
def test_attention_of_several_roots(layout):
    """Nodes without a parent see the committed keys and themselves; wide, flat trees too."""
    Case(layout, [40, 9, 300], [[-1] * 40, [-1, 0, -1, 2, 2, -1], [-1] + [0] * 30], 0, 6).check()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[3]], ids=str)
@pytest.mark.parametrize("window", [0, 128])
def test_attention_large_scores_and_sinks(layout, window):
    """Scores of hundreds, sinks of +-30, and no sinks."""
    rng = np.random.default_rng(7)
    sinks = torch.from_numpy(np.resize([30.0, -30.0, 0.5, 4.0], layout[0]).astype(np.float32))
    Case(layout, [0, 900, 47, 16], trees(rng, [12, 30, 7, 1]), window, 8, q_scale=50.0, sinks=sinks).check()
    Case(layout, [0, 900, 47, 16], trees(rng, [12, 30, 7, 1]), window, 9, sinks=None).check()


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("window", [0, 24])
def test_attention_contents_that_no_node_sees(layout, bad, window):
    """NaN and infinities in K and V behind the tree, left of every window, in free
    pages and in other branches change no bit of the nodes that do not see them; the
    nodes that do see them are not finite."""
    rng = np.random.default_rng(10)
    c = Case(layout, [75, 3], [[-1, 0, 0, 1, 1, 2, 2, 3], [-1, -1, 0, 1]], window, 11)
    clean = c.run()
    ko, vo = R.slot_offsets(c.shape.head_dim)

    def put(b, slot, what=(0, 1)):
        page = int(c.table[b, slot // PAGE])
        for i, (x, off) in enumerate(((c.k, ko), (c.v, vo))):
            if i in what:
                x[page][:, torch.from_numpy(off[slot % PAGE])] = bad

    used = set(c.table[c.table >= 0].tolist())
    for p in range(c.n_pages):
        if p not in used:
            c.k[p] = bad
            c.v[p] = bad
    for b in range(2):
        end = int(c.seq[b] + c.cu[b + 1] - c.cu[b])
        for slot in range(end, -(-end // PAGE) * PAGE):
            put(b, slot)
    if window:
        for slot in range((75 - window + 1) // PAGE * PAGE, 75 - window + 1):
            put(0, slot)
    assert torch.equal(c.run().view(torch.uint8), clean.view(torch.uint8))
    put(0, 75 + 2)          # node 2 of tree 0: seen by itself, 5 and 6
    put(1, 3 + 1, what=(1,))  # node 1 of tree 1: seen by itself and 3
    got = c.run()
    hit = np.array([2, 5, 6, 8 + 1, 8 + 3])
    rest = np.setdiff1d(np.arange(12), hit)
    assert torch.equal(got[rest].view(torch.uint8), clean[rest].view(torch.uint8))
    # a key of all -inf may give a score of -inf, whose weight is zero against values that are not finite
    assert not torch.isfinite(got[hit].float()).any()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2], LAYOUTS[3]], ids=str)
def test_attention_missing_pages(layout):
    """A missing page's keys are skipped and reported; a node without any key and without a sink gives zeros."""
    rng = np.random.default_rng(12)
    c = Case(layout, [100, 20, 5], trees(rng, [9, 4, 3]), 0, 13, sinks=None)
    c.table[0, 2] = -1
    c.table[1, 0] = c.n_pages
    c.table[2] = -1
    got = c.check(errors=mcpu.DEVERR_PAGE)
    assert (got[13:] == 0).all()


def test_attention_device_arrays_that_disagree_with_the_host():
    """Shorter lengths or other trees on the device than the host planned for set the plan's error bit; a parent
    outside its range sets the tree's, and its node counts as a root."""
    rng = np.random.default_rng(14)
    c = Case(LAYOUTS[2], [900, 40], trees(rng, [20, 8]), 0, 15)
    c.run(errors=mcpu.DEVERR_PLAN, device=dict(seq=[100, 40]))
    c.run(errors=mcpu.DEVERR_PLAN, device=dict(seq=[-5, 40]))
    c.run(errors=mcpu.DEVERR_PLAN, device=dict(cu=[0, -3, 28]))
    c.run(errors=mcpu.DEVERR_PLAN, device=dict(seq=[1 << 30, 40]))
    par = c.par.copy()
    par[5], par[22] = 7, -9
    got = c.run(errors=mcpu.DEVERR_TREE, device=dict(par=par))
    par[5] = par[22] = -1
    c.par = par
    assert torch.equal(got, c.run())


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[2]], ids=str)
def test_attention_bits_repeat_and_do_not_depend_on_placement(layout):
    rng = np.random.default_rng(16)
    c = Case(layout, [500, 33, 1200], trees(rng, [12, 64, 5]), 0, 17)
    a = c.run()
    assert torch.equal(a, c.run())
    perm = np.random.default_rng(18).permutation(c.n_pages)
    inv = np.argsort(perm)
    c.k, c.v = c.k[torch.from_numpy(perm)], c.v[torch.from_numpy(perm)]
    c.table = np.where(c.table >= 0, inv[np.maximum(c.table, 0)], -1).astype(np.int32)
    assert torch.equal(a, c.run())


def test_attention_on_another_stream_and_used_workspace():
    """On a side stream; then a smaller step with the same, no longer empty workspace."""
    rng = np.random.default_rng(19)
    c = Case(LAYOUTS[2], [2000, 10], trees(rng, [30, 9]), 0, 20)
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(c.shape, 2, c.T))
    a = c.run()
    assert torch.equal(a, c.run(ws=ws, stream=torch.cuda.Stream()))
    d = Case(LAYOUTS[2], [300], trees(rng, [7]), 0, 21)
    assert torch.equal(d.run(), d.run(ws=ws))


# Many KV heads make a batch large (more than 12288 (page, head) pairs) at a length that the 64-bit definition can
# follow: 2 x 20 to 4 x 40 columns take the staged forms of large batches, 3 the streaming one without stages.
@pytest.mark.parametrize("layout,n", [((64, 32, 64, "bf16"), 20), ((64, 32, 64, "bf16"), 50), ((128, 32, 64, "bf16"), 40),
                                      ((128, 32, 64, "bf16"), 64),
                                      ((32, 32, 64, "bf16"), 3)], ids=str)
@pytest.mark.parametrize("window", [0, 2000])
def test_attention_of_large_batches(layout, n, window):
    rng = np.random.default_rng(n)
    Case(layout, [2500, 2481, 2500 if window else 1300, 0], trees(rng, [n, n - 1, n, 1]), window, 26).check()


@pytest.mark.parametrize("layout", [(64, 4, 32, "f32"), (64, 4, 64, "f32"), (64, 4, 32, "bf16"), (64, 4, 64, "bf16")], ids=str)
def test_attention_of_many_rows_in_few_splits(layout):
    """More than 16384 (node, head) pairs in two to four splits, and a tree that is not split."""
    rng = np.random.default_rng(33)
    Case(layout, [600, 431, 900, 20, 750], trees(rng, [64, 60, 61, 62, 64]), 0, 34).check()


@pytest.mark.parametrize("layout", [LAYOUTS[0], LAYOUTS[3]], ids=str)
@pytest.mark.parametrize("longest", [300, 3000])
def test_attention_of_more_than_256_sequences(layout, longest):
    """Beyond the batch whose row offsets one workgroup scans: short trees, and some that are split."""
    rng = np.random.default_rng(longest)
    seq = rng.integers(0, 60, 301)
    seq[[7, 200, 300]] = longest
    Case(layout, seq, trees(rng, rng.integers(0, 5, 301)), 0, 27).check()


def test_attention_in_two_graphs_that_share_a_workspace():
    """Two captured calls of different batches on one workspace, replayed in turn with eager calls between them."""
    rng = np.random.default_rng(28)
    cases = [Case(LAYOUTS[2], [2000, 10], trees(rng, [30, 9]), 0, 29), Case(LAYOUTS[2], [300, 5, 900], trees(rng, [7, 64, 3]), 0, 30)]
    want = [c.run() for c in cases]
    ws = mcpu.workspace(max(mcpu.tree_attention_workspace_size(c.shape, len(c.seq), c.T) for c in cases))
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    graphs, outs, keep = [], [], []
    for c in cases:
        s = c.shape
        page = (c.n_pages, s.n_kv_heads, PAGE, s.head_dim)
        pool = mcpu.KVPool(s, c.k.cuda().view(page), c.v.cuda().view(page))
        o = torch.zeros((c.T, s.n_q_heads * s.head_dim), dtype=s.torch_dtype, device="cuda")
        args = (s, c.sinks.cuda(), pool, up(c.table), up(c.seq), up(c.cu), up(c.par), c.seq, c.cu, c.q.cuda(), o, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mcpu.tree_attention(*args)
        graphs.append(g), outs.append(o), keep.append(args)
    for i in (0, 1, 1, 0, 1, 0):
        outs[i].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i].cpu().view(want[i].shape), want[i])
        cases[1 - i].run(ws=ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0


def test_refusals_of_tensors():
    """Types, lengths, strides and devices that the calls would misread."""
    c = Case(LAYOUTS[3], [40, 9], trees(np.random.default_rng(31), [6, 4]), 0, 32)
    s, n = c.shape, c.T
    page = (c.n_pages, s.n_kv_heads, PAGE, s.head_dim)
    pool = mcpu.KVPool(s, c.k.cuda().view(page), c.v.cuda().view(page))
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(s, 2, n))
    good = dict(table=up(c.table), seq=up(c.seq), cu=up(c.cu), par=up(c.par), hseq=c.seq, hcu=c.cu, q=c.q.cuda(),
                o=torch.zeros((n, 512), dtype=torch.bfloat16, device="cuda"))
    call = lambda **kw: (lambda a: mcpu.tree_attention(s, None, pool, *a.values(), ws))({**good, **kw})  # noqa: E731
    call()
    wide = torch.zeros((n, 1024), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(seq=good["seq"].long()), dict(seq=good["seq"][:1]), dict(cu=good["cu"][:2]), dict(par=good["par"][:-1]),
                dict(par=up(np.repeat(c.par, 2))[::2]), dict(q=good["q"].float()), dict(q=good["q"][:-1]), dict(o=wide[:, :512]),
                dict(q=good["q"].cpu()), dict(seq=good["seq"].cpu()), dict(hseq=c.seq[:1]), dict(hcu=c.cu[:2]),
                dict(table=good["table"].t()), dict(o=good["o"].view(torch.float16))):
        with pytest.raises(mcpu.McpuError):
            call(**bad)
    path, two = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for i, bad in ((1, good["par"].long()), (2, good["par"][:-1]), (4, path[:-1]), (5, two[:1]), (6, two.cpu())):
        a = [good["cu"], good["par"], path, path, path.clone(), two, two.clone()]
        a[i] = bad
        with pytest.raises(mcpu.McpuError):
            mcpu.tree_accept(*a, ws)
    for i, bad in ((0, good["table"].cpu()), (1, good["seq"][:1]), (2, good["cu"].long()), (3, path.cpu()), (4, two[:1])):
        a = [good["table"], good["seq"], good["cu"], path, two]
        a[i] = bad
        with pytest.raises(mcpu.McpuError):
            mcpu.kv_tree_commit([pool], *a, ws)
    for src, hs in ((two.cpu(), [0, 0]), (two.long(), [0, 0]), (two, [0])):
        with pytest.raises(mcpu.McpuError):
            mcpu.kv_pages_copy([pool], src, two, np.array(hs, np.int32), np.array([1, 2], np.int32), ws)
    for bad in (ws.cpu(), ws[4:]):
        with pytest.raises(mcpu.McpuError):
            mcpu.tree_accept(good["cu"], good["par"], path, path, path.clone(), two, two.clone(), bad)
    for bad in (c.sinks, c.sinks[:4].cuda(), c.sinks.cuda().double()):
        with pytest.raises(mcpu.McpuError):
            mcpu.tree_attention(s, bad, pool, *good.values(), ws)
    torch.cuda.synchronize()
    assert mcpu.mcpu_check_device_errors(ws) == 0


def test_attention_pools_off_16_byte_boundaries():
    """Pools that start 8 bytes past a 16-byte boundary."""
    rng = np.random.default_rng(22)
    c = Case(LAYOUTS[2], [300, 9], trees(rng, [21, 6]), 0, 23)
    s = c.shape
    bufs = [torch.empty(x.numel() + 4, dtype=x.dtype, device="cuda") for x in (c.k, c.v)]
    k, v = (b[4:].view(c.n_pages, s.n_kv_heads, PAGE, s.head_dim) for b in bufs)
    k.copy_(c.k.view(k.shape)), v.copy_(c.v.view(v.shape))
    pool = mcpu.KVPool(s, k, v)
    o = torch.empty((c.T, s.n_q_heads * s.head_dim), dtype=s.torch_dtype, device="cuda")
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(s, 2, c.T))
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    mcpu.tree_attention(s, c.sinks.cuda(), pool, dev(c.table), dev(c.seq), dev(c.cu), dev(c.par), c.seq, c.cu,
                        c.q.cuda(), o, ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0
    ref, tol = c.reference()
    assert (np.abs(o.cpu().double().numpy().reshape(ref.shape) - ref) <= tol).all()


def test_attention_page_offsets_past_32_bits():
    """Pages whose element offsets pass 2^31: 300,000 pages of 8 KV heads (4.9 GB a pool)."""
    rng = np.random.default_rng(24)
    c = Case(LAYOUTS[2], [200], trees(rng, [20]), 0, 25)
    s, far = c.shape, 300000
    k = torch.zeros((far, s.n_kv_heads, PAGE, s.head_dim), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[-c.n_pages:] = c.k.cuda().view(-1, *k.shape[1:])
    v[-c.n_pages:] = c.v.cuda().view(-1, *k.shape[1:])
    table = np.where(c.table >= 0, c.table + far - c.n_pages, -1).astype(np.int32)
    pool = mcpu.KVPool(s, k, v)
    o = torch.empty((c.T, s.n_q_heads * s.head_dim), dtype=s.torch_dtype, device="cuda")
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(s, 1, c.T))
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    mcpu.tree_attention(s, c.sinks.cuda(), pool, dev(table), dev(c.seq), dev(c.cu), dev(c.par), c.seq, c.cu, c.q.cuda(),
                        o, ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0
    assert torch.equal(o.cpu().view(c.T, s.n_q_heads, s.head_dim), c.run())
    # commit and copy at the same offsets
    path = np.full(c.T, -1, np.int32)
    path[:3] = [0, 4, 11]
    mcpu.kv_tree_commit([pool], dev(table), dev(c.seq), dev(c.cu), dev(path), dev(np.array([3], np.int32)), ws)
    src, dst = np.array([far - 1, far - 2], np.int32), np.array([0, far - c.n_pages - 1], np.int32)
    mcpu.kv_pages_copy([pool], dev(src), dev(dst), src, dst, ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0
    ko, vo = R.slot_offsets(s.head_dim)
    for x, host, off in ((k, c.k, ko), (v, c.v, vo)):
        new = R.commit(host.float().numpy(), off, c.table, c.seq, c.cu, path, np.array([3]))
        assert (x[-c.n_pages:].cpu().float().numpy().reshape(new.shape) == new).all()
        assert torch.equal(x[0], x[-1]) and torch.equal(x[far - c.n_pages - 1], x[-2])


# ------------------------------------------------------------------------------ acceptance and commit


def _accept(cu, par, draft, sampled, errors=0):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    T, B = len(par), len(cu) - 1
    path = torch.full((T + 3,), 99, dtype=torch.int32, device="cuda")
    n_path, following = (torch.full((B + 1,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = mcpu.workspace(256)
    mcpu.tree_accept(dev(cu), dev(par), dev(draft), dev(sampled), path, n_path, following, ws)
    assert mcpu.mcpu_check_device_errors(ws) == errors
    assert (path[T:] == 99).all() and n_path[B] == 99 and following[B] == 99
    return path[:T].cpu().numpy(), n_path[:B].cpu().numpy(), following[:B].cpu().numpy()


@pytest.mark.parametrize("sizes,ids", [([1], 3), ([64] * 5, 2), ([0, 3, 64, 0, 17, 1, 40], 3), ([7] * 300, 4), ([0, 0], 1)])
def test_accept_takes_the_confirmed_path(sizes, ids):
    """Few distinct ids, so that paths are long and siblings repeat an id (the lowest is taken)."""
    rng = np.random.default_rng(sum(sizes) + ids)
    tr = trees(rng, sizes, 6)
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    par = np.array([p for t in tr for p in t], np.int32)
    draft, sampled = rng.integers(0, ids, len(par)), rng.integers(0, ids, len(par))
    for got, want in zip(_accept(cu, par, draft, sampled), R.accept(cu, par, draft, sampled)):
        np.testing.assert_array_equal(got, want)


def test_accept_chain_to_the_end_and_ids_of_any_value():
    chain = np.arange(-1, 63, dtype=np.int32)
    ids = np.array([2147483647, -2147483648, -1, 0] * 16, np.int32)
    path, n_path, following = _accept([0, 64], chain, ids, np.roll(ids, -1))
    np.testing.assert_array_equal(path, np.arange(64))
    assert n_path[0] == 64 and following[0] == ids[0]


def test_accept_reports_bad_parents_and_row_ranges():
    """A parent that does not lie before its node is never followed; a tree outside the rows has no path."""
    path, n_path, following = _accept([0, 3], [-1, 1, 0], [5, 5, 5], [5, 5, 5], errors=mcpu.DEVERR_TREE)
    np.testing.assert_array_equal(path, [0, 2, -1])
    path, n_path, following = _accept([0, 2, 9], [-1, 0], [5, 6], [6, 5], errors=mcpu.DEVERR_PLAN)
    assert n_path.tolist() == [2, 0] and following.tolist() == [5, -1]


def _paths(rng, tr):
    out, n = [], []
    for t in tr:
        at, nodes = (int(rng.integers(0, len(t))) if t else -1), []
        while at >= 0:
            nodes.append(at)
            at = t[at]
        out += nodes[::-1] + [-1] * (len(t) - len(nodes))
        n.append(len(nodes))
    return np.array(out, np.int32), np.array(n, np.int32)


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("layers", [1, 5])
def test_commit_moves_the_path_and_nothing_else(layout, layers):
    rng = np.random.default_rng(30 + layers)
    tr = trees(rng, [1, 64, 0, 5, 33, 64, 20], 3) + [[i - 1 for i in range(30)]]
    c = Case(layout, [0, 1, 15, 16, 17, 203, 31, 40], tr, 0, 31)
    s = c.shape
    page = (c.n_pages, s.n_kv_heads, PAGE, s.head_dim)
    ks = [torch.roll(c.k, i).cuda().view(page) for i in range(layers)]
    vs = [torch.roll(c.v, 3 * i + 1).cuda().view(page) for i in range(layers)]
    pools = [mcpu.KVPool(s, k, v) for k, v in zip(ks, vs)]
    path, n_path = _paths(rng, tr)
    # the shared prefix of a path and its moved part both occur; a whole chain in place too
    n_path[-1] = 30
    path[c.cu[-2]:c.cu[-1]] = np.arange(30)
    before = [x.cpu().view(c.k.shape).float().numpy() for x in ks + vs]
    ws = mcpu.workspace(256)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    mcpu.kv_tree_commit(pools, dev(c.table), dev(c.seq), dev(c.cu), dev(path), dev(n_path), ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0
    ko, vo = R.slot_offsets(s.head_dim)
    for i, x in enumerate(ks + vs):
        want = R.commit(before[i], ko if i < layers else vo, c.table, c.seq, c.cu, path, n_path)
        np.testing.assert_array_equal(x.cpu().view(c.k.shape).float().numpy(), want)


def test_commit_of_bad_paths_and_missing_pages():
    """A path that does not ascend inside its tree moves nothing; a missing page drops its tokens only."""
    chain = [i - 1 for i in range(20)]
    c = Case(LAYOUTS[3], [10, 10, 10, 10], [chain] * 4, 0, 33)
    s = c.shape
    k, v = (x.cuda().view(c.n_pages, s.n_kv_heads, PAGE, s.head_dim) for x in (c.k, c.v))
    pool = mcpu.KVPool(s, k, v)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    ws = mcpu.workspace(256)

    def run(paths, n_path, table, errors):
        path = np.full(80, -1, np.int32)
        for b, p in enumerate(paths):
            path[20 * b:20 * b + len(p)] = p
        k.copy_(c.k.cuda().view(k.shape)), v.copy_(c.v.cuda().view(v.shape))
        mcpu.kv_tree_commit([pool], dev(table), dev(c.seq), dev(c.cu), dev(path), dev(n_path), ws)
        assert mcpu.mcpu_check_device_errors(ws) == errors
        return path, np.array(n_path)

    run([[0, 2, 1], [0, 2, 2], [1, 20], [0, -1]], [3, 3, 2, 2], c.table, mcpu.DEVERR_TREE)
    assert torch.equal(k.cpu().view(c.k.shape), c.k) and torch.equal(v.cpu().view(c.v.shape), c.v)
    run([[0]] * 4, [-1, 21, 1, 0], c.table, mcpu.DEVERR_PLAN)
    assert torch.equal(k.cpu().view(c.k.shape), c.k)
    table = c.table.copy()
    table[1, 1] = -1
    table[2, 1] = c.n_pages + 5
    path, n_path = run([[0, 3, 5, 9]] * 4, [4] * 4, table, mcpu.DEVERR_PAGE)
    table[2, 1] = -1
    ko, vo = R.slot_offsets(s.head_dim)
    np.testing.assert_array_equal(k.cpu().float().numpy().reshape(c.k.shape),
                                  R.commit(c.k.float().numpy(), ko, table, c.seq, c.cu, path, n_path))
    np.testing.assert_array_equal(v.cpu().float().numpy().reshape(c.v.shape),
                                  R.commit(c.v.float().numpy(), vo, table, c.seq, c.cu, path, n_path))


# ------------------------------------------------------------------------------ page copies


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("n,layers,offset", [(1, 1, 0), (37, 3, 0), (5, 2, 4)])
def test_pages_copy(layout, n, layers, offset):
    """Repeated sources, several layers, pools off 16-byte boundaries; other pages stay as they were."""
    rng = np.random.default_rng(n)
    s = shape_of(layout)
    n_pages = 2 * n + 4
    page = (n_pages, s.n_kv_heads, PAGE, s.head_dim)
    size = int(np.prod(page))
    host = [torch.from_numpy(rng.standard_normal(page).astype(np.float32)).to(s.torch_dtype) for _ in range(2 * layers)]
    bufs = [torch.empty(size + offset, dtype=s.torch_dtype, device="cuda") for _ in host]
    dev = [b[offset:].view(page) for b in bufs]
    for d, h in zip(dev, host):
        d.copy_(h)
    pools = [mcpu.KVPool(s, dev[2 * i], dev[2 * i + 1]) for i in range(layers)]
    perm = rng.permutation(n_pages).astype(np.int32)
    src, dst = perm[rng.integers(0, max(1, n // 2), n)], np.ascontiguousarray(perm[n:2 * n])
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    ws = mcpu.workspace(256)
    mcpu.kv_pages_copy(pools, up(src), up(dst), src, dst, ws)
    assert mcpu.mcpu_check_device_errors(ws) == 0
    for d, h in zip(dev, host):
        h[torch.from_numpy(dst).long()] = h[torch.from_numpy(src).long()]
        assert torch.equal(d.cpu(), h)
    # ids that are bad on the device alone are skipped
    bad = dst.copy()
    bad[0] = n_pages
    mcpu.kv_pages_copy(pools, up(src), up(bad), src, dst, ws)
    assert mcpu.mcpu_check_device_errors(ws) == mcpu.DEVERR_PAGE
    for d, h in zip(dev, host):
        assert torch.equal(d.cpu(), h)


# ------------------------------------------------------------------------------ a step of all of them


def _step_inputs(rng, s, seq, tr, n_pages):
    T = sum(len(t) for t in tr)
    normal = lambda *shp: torch.from_numpy(rng.standard_normal(shp).astype(np.float32)).to(s.torch_dtype)  # noqa: E731
    return dict(k_new=normal(T, s.n_kv_heads, s.head_dim), v_new=normal(T, s.n_kv_heads, s.head_dim),
                q=normal(T, s.n_q_heads, s.head_dim))


def test_step_append_attend_accept_commit_and_go_on():
    """Two layers: a tree is appended, attended and accepted, its path committed, and the next token attends. The
    result equals, bit for bit, that of caches into which the path was appended token by token. The same work
    captured into a graph and replayed gives the same bits each time."""
    rng = np.random.default_rng(40)
    s = shape_of(LAYOUTS[2])
    seq = np.array([70, 14, 0], np.int32)
    tr = [R.random_tree(rng, 20, 3), R.random_tree(rng, 9, 3), R.random_tree(rng, 33, 2)]
    c = Case(LAYOUTS[2], seq, tr, 0, 41)
    page = (c.n_pages, s.n_kv_heads, PAGE, s.head_dim)
    first = [c.k.cuda().view(page), c.v.cuda().view(page), torch.roll(c.k, 5).cuda().view(page), torch.roll(c.v, 7).cuda().view(page)]
    new = [_step_inputs(rng, s, seq, tr, c.n_pages) for _ in range(2)]
    draft, sampled = rng.integers(0, 2, c.T).astype(np.int32), rng.integers(0, 2, c.T).astype(np.int32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    table, d_seq, cu, par, d_draft, d_sampled = (up(a) for a in (c.table, seq, c.cu, c.par, draft, sampled))
    new = [{k_: v_.cuda() for k_, v_ in x.items()} for x in new]
    pools_t = [x.clone() for x in first]
    pools = [mcpu.KVPool(s, pools_t[2 * i], pools_t[2 * i + 1]) for i in range(2)]
    ws = mcpu.workspace(mcpu.tree_attention_workspace_size(s, 3, c.T))
    o = [torch.empty((c.T, s.n_q_heads * s.head_dim), dtype=s.torch_dtype, device="cuda") for _ in range(2)]
    path, n_path, following = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (c.T, 3, 3))

    def step():
        for i in range(2):
            mcpu.kv_pages_append(pools[i], table, d_seq, cu, new[i]["k_new"], new[i]["v_new"], ws)
            mcpu.tree_attention(s, None, pools[i], table, d_seq, cu, par, seq, c.cu, new[i]["q"], o[i], ws)
        mcpu.tree_accept(cu, par, d_draft, d_sampled, path, n_path, following, ws)
        mcpu.kv_tree_commit(pools, table, d_seq, cu, path, n_path, ws)

    step()
    assert mcpu.mcpu_check_device_errors(ws) == 0
    want = R.accept(c.cu, c.par, draft, sampled)
    np.testing.assert_array_equal(path.cpu().numpy(), want[0])
    np.testing.assert_array_equal(n_path.cpu().numpy(), want[1])
    eager = [x.clone() for x in pools_t + o + [path, n_path, following]]
    assert max(want[1]) > 2, "the draws should confirm something"
    # token by token: the path's rows appended one after the other
    for i in range(2):
        k, v = first[2 * i].clone(), first[2 * i + 1].clone()
        pool = mcpu.KVPool(s, k, v)
        at = seq.copy()
        for j in range(int(max(want[1]))):
            rows = [int(c.cu[b] + want[0][c.cu[b] + j]) for b in range(3) if j < want[1][b]]
            who = [b for b in range(3) if j < want[1][b]]
            mcpu.kv_pages_append(pool, up(c.table[who]), up(at[who]), None, new[i]["k_new"][rows].contiguous(),
                                 new[i]["v_new"][rows].contiguous(), ws)
            at[who] += 1
        qn = new[i]["q"][:3].contiguous()
        # the last committed token is at `at - 1`; it attends in both caches
        res = []
        for p in (pool, pools[i]):
            out = torch.empty((3, s.n_q_heads * s.head_dim), dtype=s.torch_dtype, device="cuda")
            w = mcpu.workspace(mcpu.paged_attention_workspace_size(s, 3, 3))
            mcpu.paged_attention(s, None, p, table, up(at - 1), None, at - 1, None, qn, out, w)
            assert mcpu.mcpu_check_device_errors(w) == 0
            res.append(out)
        assert torch.equal(res[0], res[1])
    # captured: the graph starts from the first caches each time
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for x, y in zip(pools_t, first):
            x.copy_(y)
        step()
    for _ in range(3):
        for x in pools_t + o + [path, n_path, following]:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(pools_t + o + [path, n_path, following], eager):
            assert torch.equal(x, y)
    assert mcpu.mcpu_check_device_errors(ws) == 0
