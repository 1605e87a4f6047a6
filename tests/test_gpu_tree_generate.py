"""Trees and shared pages through the layer, the generator and the engine on
the GPU: a layer step over trees against steps over each branch alone, and
trajectories of tree steps, of groups on one prompt and of the drafting engine
against the reference's token for token (near ties as in test_gpu_generate)."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import generate as OG
from oracle import oracle as O
from paper_2608_22167_amd import mcpu, rollout, workload as W
from paper_2608_22167_amd.generate import GenSpec, Generator
from tests import parity as PT
from tests import tree_reference as R
from tests.test_gpu_generate import DELTA, LP_TOL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------ the layer


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _layer(wl, weights, k, v, seq, cu, x, table, parents=None):
    """One layer step (over trees if parents are given) on copies of the pools; o, h1, x_out and the pools."""
    s, T = wl.shape, int(cu[-1])
    k, v = k.clone(), v.clone()
    pool = mcpu.KVPool(s, k, v)
    o = torch.empty((T, s.attn_dim), dtype=s.torch_dtype, device="cuda")
    h1 = torch.empty((T, s.hidden), device="cuda")
    out = torch.empty_like(x)
    taps = mcpu.Taps(o=o.data_ptr(), h1=h1.data_ptr())
    if parents is None:
        ws = mcpu.workspace(mcpu.decode_layer_workspace_size(s, len(seq), T))
        mcpu.decode_layer(s, weights, pool, _up(table), _up(seq), _up(cu), seq, cu, x, out, taps=taps, workspace=ws)
    else:
        ws = mcpu.workspace(mcpu.decode_layer_tree_workspace_size(s, len(seq), T))
        mcpu.decode_layer_tree(s, weights, pool, _up(table), _up(seq), _up(cu), _up(parents), seq, cu, x, out, taps=taps,
                               workspace=ws)
    torch.cuda.synchronize()
    assert mcpu.mcpu_check_device_errors(ws) == 0
    return o, h1, out, k, v


@pytest.mark.parametrize("shape", [W.TINY, replace(W.GPT_OSS_20B), replace(W.GPT_OSS_20B, window=128),
                                   replace(W.GPT_OSS_20B, n_q_heads=8, n_kv_heads=2, window=7)],
                         ids=["tiny", "full", "window", "short_window"])
def test_layer_over_trees_equals_its_branches(shape):
    """Every root-to-leaf branch, run alone as a chunk, gives the rows that its nodes have in the tree step: the
    attention output and the residual behind it at the layer tolerance (the experts' choice may flip on near ties),
    and the same keys and values."""
    rng = np.random.default_rng(50)
    seq = np.array([40, 0, 17, 200], np.int32)
    tr = [R.random_tree(rng, 21, 3), R.random_tree(rng, 9, 2), [-1], R.random_tree(rng, 40, 4)]
    n = np.array([len(t) for t in tr])
    wl = W.custom(shape, seq, n, 1301, sink_std=0.5)
    cu = wl.cu_q
    par = np.array([p for t in tr for p in t], np.int32)
    weights = mcpu.DeviceWeights(shape, wl.weights)
    k, v, x = wl.k_pool.cuda(), wl.v_pool.cuda(), wl.x_in.cuda()
    o, h1, out, k1, v1 = _layer(wl, weights, k, v, seq, cu, x, wl.page_table, par)
    ko, vo = R.slot_offsets(shape.head_dim)
    done = set()
    for b, t in enumerate(tr):
        for leaf in [i for i in range(len(t)) if i not in t]:
            branch, a = [], leaf
            while a >= 0:
                branch.append(a)
                a = t[a]
            branch = branch[::-1]
            rows = [int(cu[b]) + i for i in branch]
            c = np.array([0, len(rows)], np.int32)
            o2, h2, out2, k2, v2 = _layer(wl, weights, k, v, seq[b:b + 1], c, x[rows].contiguous(), wl.page_table[b:b + 1])
            PT.check("o", o[rows].float().cpu(), o2.float().cpu(), shape.dtype)
            PT.check("h1", h1[rows].cpu(), h2.cpu(), shape.dtype)
            if shape.dtype == "f32":
                PT.check("out", out[rows].cpu(), out2.cpu(), shape.dtype)
            for depth, i in enumerate(branch):
                if (b, i) in done:
                    continue
                done.add((b, i))
                for off, one, two in ((ko, k1, k2), (vo, v1, v2)):
                    tree_slot, slot = int(seq[b]) + i, int(seq[b]) + depth
                    got = one[wl.page_table[b, tree_slot // 16]].flatten(1)[:, torch.from_numpy(off[tree_slot % 16])]
                    want = two[wl.page_table[b, slot // 16]].flatten(1)[:, torch.from_numpy(off[slot % 16])]
                    PT.check("kv", got.float().cpu(), want.float().cpu(), shape.dtype)
    assert len(done) == len(par)


def test_layer_over_trees_of_mxfp4_and_of_chains():
    """Trees that are chains are the chunks of decode_layer, here with MXFP4 experts."""
    shape = replace(W.GPT_OSS_20B, expert_fmt="mxfp4", n_experts=4, top_k=4, hidden=256, ffn_dim=256, n_q_heads=16, n_kv_heads=2)
    seq, n = np.array([33, 90, 5], np.int32), np.array([12, 1, 15])
    wl = W.custom(shape, seq, n, 1302, sink_std=0.5)
    par = np.concatenate([np.arange(-1, k - 1) for k in n]).astype(np.int32)
    weights = mcpu.DeviceWeights(shape, wl.weights)
    args = (wl, weights, wl.k_pool.cuda(), wl.v_pool.cuda(), seq, wl.cu_q, wl.x_in.cuda(), wl.page_table)
    a, b = _layer(*args, par), _layer(*args)
    for name, i in (("o", 0), ("h1", 1), ("out", 2)):
        PT.check(name, a[i].float().cpu(), b[i].float().cpu(), "bf16")
    assert torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])  # the same keys and values, bit for bit


@pytest.mark.parametrize("batch", [5, 20, 300])
def test_layer_over_many_chains(batch):
    """Up to 300 chains, whose projections take other kernels than a few rows do (and more than 256 trees)."""
    shape = replace(W.GPT_OSS_20B, n_experts=4, top_k=4, hidden=512, ffn_dim=256, n_q_heads=16, n_kv_heads=4, window=40)
    rng = np.random.default_rng(batch)
    seq = rng.integers(0, 150, batch).astype(np.int32)
    n = rng.integers(30, 65, batch) if batch < 100 else rng.integers(1, 16, batch)
    wl = W.custom(shape, seq, n, 1305, sink_std=0.5)
    par = np.concatenate([np.arange(-1, k - 1) for k in n]).astype(np.int32)
    weights = mcpu.DeviceWeights(shape, wl.weights)
    args = (wl, weights, wl.k_pool.cuda(), wl.v_pool.cuda(), seq, wl.cu_q, wl.x_in.cuda(), wl.page_table)
    a, b = _layer(*args, par), _layer(*args)
    for name, i in (("o", 0), ("h1", 1), ("out", 2)):
        PT.check(name, a[i].float().cpu(), b[i].float().cpu(), "bf16")
    assert torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])


def test_layer_over_trees_in_a_graph():
    """A captured step, replayed with other inputs in the same tensors and eager work in between."""
    shape = replace(W.GPT_OSS_20B, n_q_heads=16, n_kv_heads=2, hidden=256, ffn_dim=256, n_experts=4, top_k=2)
    rng = np.random.default_rng(51)
    seq = np.array([900, 3, 60], np.int32)
    tr = [R.random_tree(rng, 30, 3), R.random_tree(rng, 5, 2), [-1]]
    n = np.array([len(t) for t in tr])
    wl = W.custom(shape, seq, n, 1304, sink_std=0.5)
    weights = mcpu.DeviceWeights(shape, wl.weights)
    k, v = wl.k_pool.cuda(), wl.v_pool.cuda()
    pool = mcpu.KVPool(shape, k, v)
    x = wl.x_in.cuda()
    out = torch.empty_like(x)
    dev = [_up(a) for a in (wl.page_table, seq, wl.cu_q, np.concatenate(tr))]
    ws = mcpu.workspace(mcpu.decode_layer_tree_workspace_size(shape, 3, int(n.sum())))
    run = lambda: mcpu.decode_layer_tree(shape, weights, pool, *dev, seq, wl.cu_q, x, out, workspace=ws)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    first = x.clone()
    for step in range(4):
        x.copy_(first.roll(step, 0))
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out, k, v)]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((out, k, v), want):
            assert torch.equal(t, w)
    assert mcpu.mcpu_check_device_errors(ws) == 0


def test_layer_over_trees_reports_positions_past_the_rope_table():
    shape = W.TINY
    wl = W.custom(shape, [20], [8], 1303)
    weights = mcpu.DeviceWeights(shape, {k: (t[:24] if k.startswith("rope") else t) for k, t in wl.weights.items()})
    pool = mcpu.KVPool(shape, wl.k_pool.cuda(), wl.v_pool.cuda())
    x = wl.x_in.cuda()
    out = torch.empty_like(x)
    ws = mcpu.workspace(mcpu.decode_layer_tree_workspace_size(shape, 1, 8))
    run = lambda par: mcpu.decode_layer_tree(shape, weights, pool, _up(wl.page_table), _up([20]), _up([0, 8]), _up(par),  # noqa: E731
                                             np.array([20], np.int32), wl.cu_q, x, out, workspace=ws)
    run([-1] + [0] * 7)  # eight nodes, positions 20 and 21
    assert mcpu.mcpu_check_device_errors(ws) == 0
    run(np.arange(-1, 7))  # a chain: positions 20 .. 27
    assert mcpu.mcpu_check_device_errors(ws) == mcpu.DEVERR_ROPE


# ------------------------------------------------------------------------------ the generator


def _spec(**kw):
    base = W.replace(W.GPT_OSS_20B, hidden=256, n_q_heads=8, n_kv_heads=2, head_dim=64, n_experts=8, top_k=2,
                     ffn_dim=256)
    return GenSpec(**dict(dict(n_layers=4, base=base, vocab=4096, window=128, pages_full=512, pages_sw=128, max_ctx=4096), **kw))


class Reference:
    def __init__(self, spec):
        self.spec, self.ss = spec, spec.stack_spec()
        self.lw = [W.stack_weights_host(self.ss, i) for i in range(spec.n_layers)]
        self.lm = W.lm_weights_host(spec.seed, self.ss.shape_full.hidden, spec.vocab)

    def check(self, sid, tokens, samples):
        """samples (position, token, logprob) of a trajectory: each the reference's draw, outside near ties."""
        rows = OG.trajectory_rows(self.ss, self.lw, self.lm["embed"], tokens[:-1])
        pos = np.array([p for p, _, _ in samples])
        ref = O.lm_head(rows[pos - 1], self.lm["g_final"], self.lm["w_lm"], self.ss.shape_full.rms_eps,
                        self.spec.temperature, seed=self.spec.seed, seq_ids=np.full(len(pos), sid, np.int32),
                        positions=pos, want_logits=True)
        for i, (p, tok, lp) in enumerate(samples):
            assert tokens[p] == tok
            best, sc = int(ref["tokens"][i]), ref["pert"][i]
            if tok != best:
                assert sc[best] - sc[tok] <= DELTA, (sid, p, tok, best)
            else:
                assert abs(lp - ref["logprob"][i]) <= LP_TOL


def test_generator_tree_steps_draw_the_reference_trajectories():
    """Drafts made of what plain steps drew (so that paths are confirmed) with wrong branches between them, for four
    sequences whose contexts cross pages and the window; a fifth has no draft, a sixth is still being prefilled."""
    spec = _spec()
    gen = Generator(spec, max_tokens_per_step=256)
    free0 = gen.free_pages()
    rng = np.random.default_rng(60)
    prompts = {sid: rng.integers(0, spec.vocab, n).tolist() for sid, n in zip(range(5), [3, 40, 121, 14, 60])}
    plain = {}
    for sid, p in prompts.items():
        gen.add(sid, p)
    while len(plain.get(0, [])) < 40:
        for sid, (tok, _) in gen.step().items():
            plain.setdefault(sid, []).append(tok)
    for sid in prompts:
        gen.release(sid)
    for sid, p in prompts.items():
        gen.add(sid, p)
    out, steps = {sid: [] for sid in prompts}, 0
    for sid, (tok, lp) in gen.step().items():
        out[sid].append((tok, lp))
    while min(len(o) for o in out.values()) < 25:
        if steps == 2:
            gen.add(7, rng.integers(0, spec.vocab, 30).tolist())  # not decoding: tree steps leave it alone
        drafts = {}
        for sid in range(4):
            known = plain[sid][len(out[sid]):len(out[sid]) + 3]
            tokens, parents, end = [], [], -1
            for t in known:
                tokens += [(t + 1) % spec.vocab, t, (t + 2) % spec.vocab]
                parents += [end] * 3
                end = len(tokens) - 2
            drafts[sid] = (tokens, parents)
        for sid, drawn in gen.step_tree(drafts).items():
            out[sid] += drawn
        steps += 1
        assert gen.check_errors() == 0
    assert 7 in gen.seqs and gen.seqs[7].length == 0 and len(gen.seqs[7].pending) == 30
    assert len(out[4]) == steps + 1                     # no draft: one token a step
    assert sum(len(out[sid]) > 2 * steps for sid in range(4)) >= 3, "drafts of the true tokens should be confirmed"
    ref = Reference(spec)
    for sid, p in prompts.items():
        s = gen.seqs[sid]
        tokens = s.history + s.pending
        assert tokens == p + [t for t, _ in out[sid]] and s.length == len(s.history)
        ref.check(sid, tokens, [(len(p) + i, t, lp) for i, (t, lp) in enumerate(out[sid])])
    for sid in list(gen.seqs):
        gen.release(sid)
    assert gen.free_pages() == free0, "pages leaked"


@pytest.mark.parametrize("length", [1, 2, 17, 33, 150])
def test_generator_group_shares_its_prompt(length):
    """Members of a group draw the reference's tokens for their own ids; whole prompt pages are held once."""
    spec = _spec(seed=3007)
    gen = Generator(spec, max_tokens_per_step=64)
    free0 = gen.free_pages()
    prompt = np.random.default_rng(length).integers(0, spec.vocab, length).tolist()
    sids = [11, 5, 8, 30]
    gen.add_group(sids, prompt)
    whole, part = (length - 1) // 16, (length - 1) % 16 > 0
    assert free0[0] - gen.free_pages()[0] == whole + len(sids) * part
    lo = max(0, length - 1 - 127) // 16
    assert free0[1] - gen.free_pages()[1] == whole - lo + len(sids) * part
    if whole:
        assert mcpu.kv_page_holders(gen.alloc_full, gen.seqs[5].pages_full[0]) == len(sids)
    out = {sid: [] for sid in sids}
    for _ in range(6):
        for sid, (tok, lp) in gen.step().items():
            out[sid].append((tok, lp))
    assert gen.check_errors() == 0
    ref = Reference(spec)
    for sid in sids:
        ref.check(sid, prompt + [t for t, _ in out[sid]], [(length + i, t, lp) for i, (t, lp) in enumerate(out[sid])])
    assert len({tuple(t for t, _ in o) for o in out.values()}) == len(sids)
    for i, sid in enumerate(sids):
        gen.release(sid)
        if whole and i < 3:
            assert mcpu.kv_page_holders(gen.alloc_full, gen.seqs[sids[3]].pages_full[0]) == 3 - i
    assert gen.free_pages() == free0


def test_generator_drafts_that_do_not_fit_are_not_tried():
    """Too few pages, or positions past the last one: such a step draws one token, the one that step() draws."""
    spec = _spec(seed=3009, pages_full=9, pages_sw=9, max_ctx=128)
    gen = Generator(spec, max_tokens_per_step=256)
    prompt = np.random.default_rng(71).integers(0, spec.vocab, 100).tolist()
    drawn = []
    for tree in (False, True):
        gen.add(0, prompt)
        out = [t for t, _ in [gen.step()[0]]]
        while len(out) < 29:  # token k of them sits at position 99 + k; the last one fed is number 28, at 127
            if tree:
                # 60 siblings need a tenth page; a chain of 20 behind token 9 or later passes position 127
                n, chain = (60, False) if len(out) < 9 else (20, True)
                known = (drawn[0][len(out):] + [1] * n)[:n]
                got = gen.step_tree({0: (known, list(range(-1, n - 1)) if chain else [-1] * n)})[0]
                assert len(got) == 1
                out += [t for t, _ in got]
            else:
                out.append(gen.step()[0][0])
        assert gen.check_errors() == 0
        drawn.append(out)
        with pytest.raises(mcpu.McpuError):  # position 128
            gen.step_tree({}) if tree else gen.step()
        gen.release(0)
    assert drawn[0] == drawn[1]
    assert gen.free_pages() == (9, 9)


def test_generator_fork_in_mid_trajectory_and_when_pages_run_out():
    spec = _spec(seed=3008, pages_full=24, pages_sw=24)
    gen = Generator(spec, max_tokens_per_step=256)
    free0 = gen.free_pages()
    prompt = np.random.default_rng(70).integers(0, spec.vocab, 200).tolist()
    gen.add(0, prompt)
    for _ in range(5):
        gen.step()
    before, free1 = (gen.seqs[0].length, list(gen.seqs[0].pending), list(gen.seqs[0].pages_full)), gen.free_pages()
    with pytest.raises(mcpu.McpuError):
        gen.fork(0, list(range(1, 30)))  # 29 last pages where fewer are left
    assert (gen.seqs[0].length, gen.seqs[0].pending, gen.seqs[0].pages_full) == before and gen.free_pages() == free1
    assert list(gen.seqs) == [0] and mcpu.kv_page_holders(gen.alloc_full, before[2][0]) == 1
    for bad in ([0], [3, 3]):
        with pytest.raises(ValueError):
            gen.fork(0, bad)
    gen.fork(0, [1, 2])
    gen.hold(1)
    gen.fork(1, [4])
    gen.resume(4, [17, 18])
    drawn = {}
    for _ in range(4):
        for sid, (tok, lp) in gen.step().items():
            drawn.setdefault(sid, []).append((tok, lp))
    assert gen.check_errors() == 0
    ref = Reference(spec)
    tokens = {sid: s.history + s.pending for sid, s in gen.seqs.items()}
    assert tokens[0][:205] == tokens[2][:205] == tokens[4][:205] and tokens[4][205:207] == [17, 18]
    # the draws after the fork are each member's own
    for sid, first in ((0, 205), (2, 205), (4, 207)):
        assert [t for t, _ in drawn[sid]] == tokens[sid][first:]
        ref.check(sid, tokens[sid], [(first + i, t, lp) for i, (t, lp) in enumerate(drawn[sid])])
    for sid in list(gen.seqs):
        gen.release(sid)
    assert gen.free_pages() == free0


def test_engine_drafts_from_history():
    """Greedy draws of a small stack soon repeat themselves, so drafts from a sequence's history are confirmed: the
    engine returns turns of the asked length, the reference's tokens, in fewer steps than tokens."""
    spec = _spec(seed=3009, temperature=0.0)
    gen = Generator(spec, max_tokens_per_step=256)
    free0 = gen.free_pages()
    rng = np.random.default_rng(80)
    prompts = {sid: np.tile(rng.integers(0, spec.vocab, 6), 4).tolist() for sid in range(3)}
    eng = rollout.Engine(gen, draft_nodes=12)
    try:
        turns = {sid: [eng.generate(sid, p, 40)] for sid, p in prompts.items()}
        obs = {sid: rng.integers(0, spec.vocab, 9).tolist() for sid in prompts}
        for sid in prompts:
            turns[sid][0] = turns[sid][0].result(timeout=100)
            turns[sid].append(eng.generate(sid, obs[sid], 15).result(timeout=100))
        assert gen.check_errors() == 0
        ref = Reference(spec)
        for sid, p in prompts.items():
            assert [len(t) for t in turns[sid]] == [40, 15]
            tokens = p + [t for t, _ in turns[sid][0]] + obs[sid] + [t for t, _ in turns[sid][1]]
            at = [len(p) + i for i in range(40)] + [len(p) + 49 + i for i in range(15)]
            ref.check(sid, tokens, [(q, t, lp) for q, (t, lp) in zip(at, turns[sid][0] + turns[sid][1])])
        print(f"  {eng.tokens} tokens in {eng.steps} steps")
        for sid in prompts:
            eng.release(sid).result(timeout=100)
    finally:
        eng.close()
    assert gen.free_pages() == free0


def test_layer_over_trees_with_native_mxfp4_experts():
    """The layer's feed-forward half on the residual that its attention left is moe_forward's, bit for bit, and the
    attention half is that of the same trees' branches (here chains) in decode_layer."""
    shape = replace(W.GPT_OSS_20B, expert_fmt="mxfp4_native", n_experts=4, top_k=2, hidden=256, ffn_dim=256,
                    n_q_heads=16, n_kv_heads=2)
    rng = np.random.default_rng(52)
    seq = np.array([33, 90, 5], np.int32)
    for tr in ([R.random_tree(rng, 12, 3), [-1], R.random_tree(rng, 40, 4)], [[i - 1 for i in range(k)] for k in (12, 1, 15)]):
        wl = W.custom(shape, seq, np.array([len(t) for t in tr]), 1306, sink_std=0.5)
        par = np.array([p for t in tr for p in t], np.int32)
        weights = mcpu.DeviceWeights(shape, wl.weights)
        args = (wl, weights, wl.k_pool.cuda(), wl.v_pool.cuda(), seq, wl.cu_q, wl.x_in.cuda(), wl.page_table)
        o, h1, out, k, v = _layer(*args, par)
        want = torch.empty_like(out)
        ws = mcpu.workspace(mcpu.moe_forward_workspace_size(shape, len(par)))
        mcpu.moe_forward(shape, weights, h1, want, workspace=ws)
        assert mcpu.mcpu_check_device_errors(ws) == 0
        assert torch.equal(out, want)
    b = _layer(*args)
    PT.check("o", o.float().cpu(), b[0].float().cpu(), "bf16")
    PT.check("h1", h1.cpu(), b[1].cpu(), "bf16")
    assert torch.equal(k, b[3]) and torch.equal(v, b[4])


def test_layer_over_trees_with_empty_trees():
    """Sequences without nodes at either end and in between change no bit of the others."""
    shape = replace(W.GPT_OSS_20B, n_q_heads=16, n_kv_heads=2, hidden=256, ffn_dim=256, n_experts=4, top_k=2)
    rng = np.random.default_rng(53)
    tr = [R.random_tree(rng, 9, 3), R.random_tree(rng, 30, 4)]
    seq, n = np.array([40, 700], np.int32), np.array([9, 30])
    wl = W.custom(shape, seq, n, 1307, sink_std=0.5)
    par = np.array([p for t in tr for p in t], np.int32)
    weights = mcpu.DeviceWeights(shape, wl.weights)
    pools_x = wl.k_pool.cuda(), wl.v_pool.cuda()
    a = _layer(wl, weights, *pools_x, seq, wl.cu_q, wl.x_in.cuda(), wl.page_table, par)
    rows = [0, 0, 1, 1, 1]
    table = wl.page_table[rows].copy()
    table[[0, 2, 4]] = -1
    cu = np.array([0, 0, 9, 9, 39, 39], np.int32)
    b = _layer(wl, weights, *pools_x, np.array([5, 40, 0, 700, 9000], np.int32), cu, wl.x_in.cuda(), table, par)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
