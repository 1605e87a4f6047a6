"""Drafted token trees over the paged KV cache, and the copying of its pages.

Four operators, each in its plain form (elementary torch operations in 32 bits)
and as the framework's call:

  attn    attention of a tree of drafted tokens over committed keys and its own
          branch (tree_attention)
  accept  the path of drafted tokens that the draws confirm (tree_accept)
  commit  the accepted path's K and V moved onto consecutive slots, in every
          layer of a kind (kv_tree_commit)
  copy    pages copied into other pages, in every layer of a kind
          (kv_pages_copy)

A case is a dict of plain values. Lengths, tree shapes and page placement follow
from its `lens`; cached keys and values, queries and token ids from the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
VOCAB = 201088
# query heads, KV heads, head dim, type: the gpt-oss-20b-shaped layer, the reduced bf16 stack that the
# generator is tested with, and the tiny fp32 layer
HEADS = {"full": (64, 8, 64, "bf16"), "reduced": (8, 2, 64, "bf16"), "tiny": (8, 2, 32, "f32")}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------


def _attn(name, heads, batch, ctx, cap, lo, hi, window=0, lens=1):
    c = dict(kind="attn", heads=heads, batch=batch, ctx=ctx, cap=cap, lo=lo, hi=hi, window=window, lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: the tiny fp32 layer, three short sequences
        _attn("tree_f32_b3", "tiny", 3, 100, 256, 1, 9, lens=101),
        # one trajectory left in flight, sixteen drafted tokens: latency, splits of one context
        _attn("tree_full_b1", "full", 1, 6000, 6000, 16, 16, lens=102),
        # a decode batch with short drafts on a full-attention layer
        _attn("tree_full_b48", "full", 48, 4096, 16384, 1, 8, lens=103),
        # a large batch on a sliding-window layer
        _attn("tree_window_b256", "full", 256, 4096, 32768, 2, 12, window=128, lens=104),
        # few sequences with the widest trees behind long contexts
        _attn("tree_full_wide_b16", "full", 16, 8192, 16384, 33, 64, lens=105),
        # the reduced stack of the generator's tests, odd sizes
        _attn("tree_reduced_b21", "reduced", 21, 700, 4096, 1, 27, lens=106),
        # a few trajectories verified
        dict(kind="accept", name="accept_b5", batch=5, lo=1, hi=16, lens=111),
        # the whole batch of the 24-layer stack, widest trees
        dict(kind="accept", name="accept_b512", batch=512, lo=1, hi=64, lens=112),
        # a few accepted tokens in the tiny fp32 layer's cache
        dict(kind="commit", name="commit_f32_b3", heads="tiny", layers=1, batch=3, lo=2, hi=9, lens=121),
        # the twelve layers of one kind of the 24-layer stack, a decode batch
        dict(kind="commit", name="commit_12_layers_b48", heads="full", layers=12, batch=48, lo=1, hi=16, lens=122),
        # groups forked from their prompts: each member gets its own last page, twelve layers
        dict(kind="copy", name="fork_12_layers_p112", heads="full", layers=12, pages=112, spare=16, lens=131),
        # whole contexts copied, two layers
        dict(kind="copy", name="copy_2_layers_p1500", heads="full", layers=2, pages=1500, spare=77, lens=132),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the listed kinds with sizes spread over their ranges."""
    kind = rng.choice(["attn", "attn", "attn", "accept", "commit", "copy"])
    lens = rng.randrange(1, 1 << 20)
    if kind == "attn":
        heads = rng.choice(["full", "full", "reduced", "tiny"])
        hi = _log_uniform(rng, 1, 64)
        lo = rng.randrange(0, hi + 1)
        if heads == "tiny":
            return _attn(None, heads, rng.randrange(1, 17), _log_uniform(rng, 1, 300), 600, lo, max(hi, 1), rng.choice([0, 128]), lens)
        batch = _log_uniform(rng, 1, 256)
        ctx = _log_uniform(rng, 1, min(8192, 200000 // batch))
        return _attn(None, heads, batch, ctx, min(16384, 4 * ctx + 16), lo, max(hi, 1), rng.choice([0, 0, 128]), lens)
    if kind == "accept":
        hi = _log_uniform(rng, 1, 64)
        return dict(kind=kind, batch=_log_uniform(rng, 1, 512), lo=rng.randrange(0, hi + 1), hi=hi, lens=lens)
    heads = rng.choice(["full", "full", "reduced", "tiny"])
    if kind == "commit":
        hi = _log_uniform(rng, 1, 64)
        return dict(kind=kind, heads=heads, layers=rng.randrange(1, 13), batch=_log_uniform(rng, 1, 48),
                    lo=rng.randrange(0, hi + 1), hi=hi, lens=lens)
    layers = rng.randrange(1, 13)
    return dict(kind=kind, heads=heads, layers=layers, pages=_log_uniform(rng, 1, 1500 // layers), spare=rng.randrange(0, 100),
                lens=lens)


# ---------------------------------------------------------------------------
# lengths, trees and placement (from the case alone)
# ---------------------------------------------------------------------------


def _trees(case, rng):
    """Node counts, their running sum and parents: node 0 is the root, a later node's parent one of the
    few before it (drafts are chains with side branches). A tree may have no node, and one node stands for a
    sequence without a draft. Of twenty trees one has a second root."""
    n = rng.integers(case["lo"], case["hi"] + 1, size=case["batch"])
    n[0] = max(n[0], 1)
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    par = np.full(int(cu[-1]), -1, np.int32)
    for b in range(case["batch"]):
        reach = int(rng.integers(1, 6))
        second = int(rng.integers(1, 65)) if rng.random() < 0.05 and case["kind"] == "attn" else 0
        for i in range(1, int(n[b])):
            if i != second:
                par[cu[b] + i] = rng.integers(max(0, i - reach), i)
    return cu, par


def _lengths(case, rng):
    """Committed tokens: log-normal around `ctx` (sigma 1), up to `cap`; a lone sequence has exactly `ctx`."""
    if case["batch"] == 1:
        return np.array([case["ctx"]], np.int32)
    x = np.exp(rng.normal(math.log(case["ctx"]), 1.0, size=case["batch"]))
    return np.clip(np.round(x), 0, case["cap"]).astype(np.int32)


def _pages(first, last, rng):
    """A table with random placement for logical pages first .. last - 1 of each sequence, in a pool a
    quarter larger than needed; other entries are -1 (freed, or not there yet)."""
    need = int((last - first).sum())
    n_pages = need + need // 4 + 1
    perm = rng.permutation(n_pages)[:need].astype(np.int32)
    table = np.full((len(first), max(1, int(last.max()))), -1, np.int32)
    at = 0
    for b in range(len(first)):
        n = int(last[b] - first[b])
        table[b, first[b]:last[b]] = perm[at:at + n]
        at += n
    return table, n_pages


def _layout(case):
    """Everything about a case's attn, accept or commit that its seed does not change."""
    rng = np.random.default_rng(case["lens"])
    cu, par = _trees(case, rng)
    n = np.diff(cu)
    if case["kind"] == "accept":
        return cu, par, None, None, None, 0
    if case["kind"] == "commit":
        # a window layer's table: only the last pages are there
        seq = rng.integers(0, 600, size=case["batch"]).astype(np.int32)
        window = 128
    else:
        seq, window = _lengths(case, rng), case["window"]
    first = (np.maximum(0, seq.astype(np.int64) - window + 1) if window else np.zeros(len(seq), np.int64)) // PAGE
    last = np.maximum((seq.astype(np.int64) + n + PAGE - 1) // PAGE, first)
    table, n_pages = _pages(first, last, rng)
    return cu, par, seq, first, table, n_pages


def _copy_ids(case):
    rng = np.random.default_rng(case["lens"])
    n_pages = 2 * case["pages"] + case["spare"]
    perm = rng.permutation(n_pages).astype(np.int32)
    # members of a group copy the same page: sources repeat, destinations do not
    src = perm[:case["pages"]][rng.integers(0, max(1, case["pages"] // 2), size=case["pages"])]
    return src, np.ascontiguousarray(perm[case["pages"]:2 * case["pages"]]), n_pages


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _torch_type(heads):
    return torch.bfloat16 if HEADS[heads][3] == "bf16" else torch.float32


# ---------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------


def _shape(case):
    from paper_2608_22167_amd import workload as W
    hq, hkv, d, t = HEADS[case["heads"]]
    return W.replace(W.TINY if t == "f32" else W.GPT_OSS_20B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
                     window=case.get("window", 0))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    if case["kind"] == "accept":
        cu, par, *_ = _layout(case)
        st.update(cu=_dev(cu), par=_dev(par), **_tokens(cu, par, seed))
        st["out"] = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (len(par), case["batch"], case["batch"])]
        if own:
            from paper_2608_22167_amd import mcpu
            st["ws"] = mcpu.workspace(256)
        return st
    hq, hkv, d, _ = HEADS[case["heads"]]
    t = _torch_type(case["heads"])
    layers = case.get("layers", 1)
    if case["kind"] == "copy":
        src, dst, n_pages = _copy_ids(case)
        st.update(src=_dev(src), dst=_dev(dst), host_src=src, host_dst=dst)
    else:
        cu, par, seq, first, table, n_pages = _layout(case)
        st.update(cu=_dev(cu), par=_dev(par), seq=_dev(seq), table=_dev(table), host_cu=cu, host_seq=seq, first=_dev(first))
    # a layer's pools are pages of [KV heads][16 slots x head dim] in the cache's own order
    st["k"] = torch.randn((layers, n_pages, hkv, PAGE, d), generator=g, device="cuda", dtype=torch.float32).to(t)
    st["v"] = torch.randn((layers, n_pages, hkv, PAGE, d), generator=g, device="cuda", dtype=torch.float32).to(t)
    if case["kind"] == "attn":
        T = len(par)
        st["q"] = (torch.randn((T, hq, d), generator=g, device="cuda") * 1.5).to(t)
        st["sinks"] = torch.randn((hq,), generator=g, device="cuda")
        st["o"] = torch.empty((T, hq * d), dtype=t, device="cuda")
        st["span"] = max(1, int(((seq.astype(np.int64) + np.diff(cu) + PAGE - 1) // PAGE - first).max()))
        st["most"] = max(1, int(np.diff(cu).max()))
    if case["kind"] == "commit":
        path, n_path = _paths(cu, par, seed)
        st.update(path=_dev(path), n_path=_dev(n_path))
    if own:
        from paper_2608_22167_amd import mcpu
        shape = st["shape"] = _shape(case)
        st["pools"] = [mcpu.KVPool(shape, st["k"][i], st["v"][i]) for i in range(layers)]
        st["ws"] = mcpu.workspace(mcpu.tree_attention_workspace_size(shape, case["batch"], len(par))
                                  if case["kind"] == "attn" else 256)
    return st


def _tokens(cu, par, seed):
    """Drafted ids and draws: a draw repeats the id of one of the node's children in three cases of four."""
    rng = np.random.default_rng([seed, 7])
    T = len(par)
    draft = rng.integers(0, VOCAB, T).astype(np.int32)
    sampled = rng.integers(0, VOCAB, T).astype(np.int32)
    for b in range(len(cu) - 1):
        for i in range(cu[b], cu[b + 1]):
            if par[i] >= 0 and rng.random() < 0.75:
                sampled[cu[b] + par[i]] = draft[i]
            if i > cu[b] and par[i] == par[i - 1] and rng.random() < 0.2:  # siblings with the same id
                draft[i] = draft[i - 1]
    return dict(draft=_dev(draft), sampled=_dev(sampled), host_draft=draft, host_sampled=sampled)


def _paths(cu, par, seed):
    """An accepted path per tree: a random node's ancestors and itself, then -1."""
    rng = np.random.default_rng([seed, 8])
    path = np.full(len(par), -1, np.int32)
    n_path = np.zeros(len(cu) - 1, np.int32)
    for b in range(len(cu) - 1):
        n = int(cu[b + 1] - cu[b])
        at = int(rng.integers(0, n)) if n else -1
        nodes = []
        while at >= 0:
            nodes.append(at)
            at = int(par[cu[b] + at])
        path[cu[b]:cu[b] + len(nodes)] = nodes[::-1]
        n_path[b] = len(nodes)
    return path, n_path


# ---------------------------------------------------------------------------
# run
# ---------------------------------------------------------------------------


def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2608_22167_amd import mcpu
        if kind == "attn":
            mcpu.tree_attention(st["shape"], st["sinks"], st["pools"][0], st["table"], st["seq"], st["cu"], st["par"],
                                st["host_seq"], st["host_cu"], st["q"], st["o"], st["ws"])
            return st["o"]
        if kind == "accept":
            path, n_path, following = st["out"]
            mcpu.tree_accept(st["cu"], st["par"], st["draft"], st["sampled"], path, n_path, following, st["ws"])
            return path, n_path, following
        if kind == "commit":
            mcpu.kv_tree_commit(st["pools"], st["table"], st["seq"], st["cu"], st["path"], st["n_path"], st["ws"])
            return st["k"], st["v"]
        mcpu.kv_pages_copy(st["pools"], st["src"], st["dst"], st["host_src"], st["host_dst"], st["ws"])
        return st["k"], st["v"]
    return dict(attn=_plain_attn, accept=_plain_accept, commit=_plain_commit, copy=_plain_copy)[kind](st)


def _ancestors(par):
    """par [B, N] (own index where a node has no parent or is not there) -> [B, N, N]: is j an ancestor of
    i, or i itself? (1 + parent matrix)^63 counts the ways down from it in at most 63 steps."""
    n = par.shape[1]
    step = torch.nn.functional.one_hot(par, n).float()
    at = torch.arange(n, device=par.device)
    step = step * (par != at).unsqueeze(2) + torch.eye(n, device=par.device)
    return torch.matrix_power(step, 63) > 0


def _nodes(cu, par, most):
    """Trees as rows of `most` nodes: token index, whether it is there, and the parent (own index: none)."""
    at = torch.arange(most, device=cu.device)
    there = at < (cu[1:] - cu[:-1]).unsqueeze(1)
    tok = torch.where(there, cu[:-1].unsqueeze(1) + at, 0).long()
    p = torch.where(there, par[tok].long(), -1)
    return tok, there, torch.where(p < 0, at, p)


def _plain_attn(st):
    case = st["case"]
    hq, hkv, d, _ = HEADS[case["heads"]]
    G, W, most = hq // hkv, case["window"], st["most"]
    tok, there, par = _nodes(st["cu"], st["par"], most)
    B = tok.shape[0]
    anc = _ancestors(par)
    depth = anc.sum(2) - 1
    # the sequences' pages side by side, from the first that is there
    pages = st["first"].unsqueeze(1) + torch.arange(st["span"], device="cuda")
    ids = st["table"].gather(1, pages.clamp(max=st["table"].shape[1] - 1)).clamp(min=0).long()
    L = st["span"] * PAGE
    k = st["k"][0][ids].view(B, -1, hkv, d // 8, PAGE, 8).permute(0, 2, 1, 4, 3, 5).reshape(B, hkv, L, d).float()
    v = st["v"][0][ids].view(B, -1, hkv, d // 16, 4, 16, 4).permute(0, 2, 1, 4, 6, 3, 5).reshape(B, hkv, L, d).float()
    q = st["q"][tok].float().view(B, most, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, most * G, d)
    # key at slot j: committed, or node j - seq
    slot = st["first"].unsqueeze(1) * PAGE + torch.arange(L, device="cuda")
    seq = st["seq"].long().unsqueeze(1)
    node = (slot - seq).clamp(0, most - 1)
    pos = seq + depth
    here = anc.gather(2, node.unsqueeze(1).expand(B, most, L)) & (slot - seq < most).unsqueeze(1)
    key_pos = torch.where(slot < seq, slot, seq + depth.gather(1, node))
    seen = torch.where((slot < seq).unsqueeze(1), torch.ones_like(here), here)
    if W:
        seen = seen & (key_pos.unsqueeze(1) > pos.unsqueeze(2) - W)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, hkv, most, G, L) * (1.0 / math.sqrt(d))
    z = z.masked_fill(~seen.view(B, 1, most, 1, L), -math.inf)
    sink = st["sinks"].view(1, hkv, 1, G, 1)
    m = torch.maximum(z.amax(4, keepdim=True), sink)
    e = torch.exp(z - m)
    total = e.sum(4, keepdim=True) + torch.exp(sink - m)
    o = torch.matmul((e / total).view(B, hkv, most * G, L), v)
    o = o.view(B, hkv, most, G, d).permute(0, 2, 1, 3, 4).reshape(B, most, hq * d)
    out = torch.empty_like(st["o"])
    row = torch.arange(out.shape[0], device="cuda")
    b = torch.searchsorted(st["cu"][1:].long().contiguous(), row, right=True)
    out.copy_(o[b, row - st["cu"][b].long()])
    return out


def _plain_accept(st):
    case = st["case"]
    most = max(1, case["hi"])
    cu = st["cu"]
    T = st["par"].numel()
    tok, there, par = _nodes(cu, st["par"], most)
    at = torch.arange(most, device="cuda")
    child = there & (par != at)
    draft = st["draft"][tok]
    hit = child & (draft == st["sampled"][tok].gather(1, par))
    # of several confirmed children of one node the lowest
    earlier = (par.unsqueeze(2) == par.unsqueeze(1)) & hit.unsqueeze(1) & (at.unsqueeze(0) < at.unsqueeze(1))
    step = (hit & ~earlier.any(2)) | ((at == 0) & there)
    anc = _ancestors(par)
    taken = there & (step.unsqueeze(1) | ~anc).all(2)
    n_path = taken.sum(1)
    order = torch.where(taken, at, most).sort(1).values
    path = torch.where(order < most, order, -1)
    last = order.gather(1, (n_path - 1).clamp(min=0).unsqueeze(1)).clamp(max=most - 1)
    following = torch.where(n_path > 0, st["sampled"][tok].gather(1, last).squeeze(1), -1)
    row = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].long().contiguous(), row, right=True)
    return path[b, row - cu[b].long()].int(), n_path.int(), following.int()


def _plain_commit(st):
    hq, hkv, d, _ = HEADS[st["case"]["heads"]]
    layers, n_pages = st["k"].shape[:2]
    cu, T = st["cu"], st["path"].numel()
    row = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].long().contiguous(), row, right=True)
    i = row - cu[b].long()
    # nodes past the path keep their place
    node = torch.where(i < st["n_path"][b], st["path"].long(), i)
    src, dst = st["seq"][b].long() + node, st["seq"][b].long() + i
    ps, pd = st["table"][b, src // PAGE].long(), st["table"][b, dst // PAGE].long()
    ss, sd = src % PAGE, dst % PAGE
    k = st["k"].view(layers, n_pages, hkv, d // 8, PAGE, 8)
    k[:, pd, :, :, sd] = k[:, ps, :, :, ss]
    v = st["v"].view(layers, n_pages, hkv, d // 16, 4, 16, 4)
    v[:, pd, :, :, sd // 4, :, sd % 4] = v[:, ps, :, :, ss // 4, :, ss % 4]
    return st["k"], st["v"]


def _plain_copy(st):
    src, dst = st["src"].long(), st["dst"].long()
    st["k"][:, dst] = st["k"][:, src]
    st["v"][:, dst] = st["v"][:, src]
    return st["k"], st["v"]


# ---------------------------------------------------------------------------
# work and exact
# ---------------------------------------------------------------------------


def _size(case):
    return 2 if HEADS[case["heads"]][3] == "bf16" else 4


def work(case):
    if case["kind"] == "accept":
        cu, *_ = _layout(case)
        return {"bytes": 4 * (4 * int(cu[-1]) + 3 * case["batch"] + 1), "flops": 0}
    hq, hkv, d, _ = HEADS[case["heads"]]
    row = hkv * d * _size(case)  # K or V of a token in one layer
    if case["kind"] == "copy":
        return {"bytes": 4 * case["layers"] * case["pages"] * PAGE * row + 8 * case["pages"], "flops": 0}
    cu, par, seq, first, table, _ = _layout(case)
    if case["kind"] == "commit":
        # about half of the nodes lie on a path, those before the first side branch in place already
        path, n_path = _paths(cu, par, 0)
        return {"bytes": 4 * case["layers"] * int(n_path.sum()) * row + 4 * int(cu[-1]) + 16 * case["batch"], "flops": 0}
    n = np.diff(cu)
    W = case["window"]
    keys = pairs = 0
    for b in range(case["batch"]):
        depth = []
        for i in range(int(n[b])):
            p = int(par[cu[b] + i])
            depth.append(0 if p < 0 else depth[p] + 1)
            own_keys, old = depth[i] + 1, int(seq[b])
            if W:
                own_keys, old = min(own_keys, W), min(old, max(0, W - depth[i] - 1))
            pairs += own_keys + old
        if n[b]:
            keys += int(n[b]) + (min(int(seq[b]), W - 1) if W else int(seq[b]))
    T = int(cu[-1])
    return {"bytes": 2 * keys * row + 2 * T * hq * d * _size(case) + 4 * table.size + 8 * T, "flops": 4 * hq * d * pairs}


def exact(case, seed):
    """From the definitions: sequence by sequence, slot by slot, in 64 bits."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return dict(attn=_exact_attn, accept=_exact_accept, commit=_exact_commit, copy=_exact_copy)[case["kind"]](st)


def _slot_index(d):
    """Element offsets of (slot, dim) within a page's K and V of one KV head."""
    s, i = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    return ((i // 8) * PAGE + s) * 8 + i % 8, (((i // 16) * 4 + s // 4) * 16 + i % 16) * 4 + s % 4


def _exact_attn(st):
    case = st["case"]
    hq, hkv, d, _ = HEADS[case["heads"]]
    G, W = hq // hkv, case["window"]
    ko, vo = (_dev(a) for a in _slot_index(d))
    cu, seq, par = st["host_cu"], st["host_seq"], st["par"].cpu().numpy()
    table, first = st["table"].cpu().numpy(), st["first"].cpu().numpy()
    kp, vp = (st[x][0].reshape(-1, hkv, PAGE * d) for x in ("k", "v"))
    out = torch.zeros((len(par), hq * d), dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        n, L = int(cu[b + 1] - cu[b]), int(seq[b])
        if n == 0:
            continue
        f = int(first[b])
        ids = _dev(table[b, f:(L + n - 1) // PAGE + 1].astype(np.int64))
        K = kp[ids][:, :, ko].double().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :L + n - f * PAGE]
        V = vp[ids][:, :, vo].double().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :L + n - f * PAGE]
        see = np.zeros((n, L + n), bool)
        depth = np.zeros(n, np.int64)
        for i in range(n):
            chain, a = [], i
            while a >= 0:
                chain.append(a)
                a = int(par[cu[b] + a])
            depth[i] = len(chain) - 1
            lo = max(0, L + depth[i] - W + 1) if W else 0
            see[i, lo:L] = True
            for back, a in enumerate(chain):
                see[i, L + a] = not W or back < W
        q = st["q"][cu[b]:cu[b + 1]].double().view(n, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, n * G, d)
        z = (q @ K.transpose(1, 2).contiguous() / math.sqrt(d)).view(hkv, n, G, -1)
        z = torch.where(_dev(see[:, f * PAGE:])[None, :, None, :], z, torch.full_like(z, -math.inf))
        z = torch.cat([z, st["sinks"].double().view(hkv, 1, G, 1).expand(hkv, n, G, 1)], 3)
        w = torch.softmax(z, 3)[..., :-1].reshape(hkv, n * G, -1)
        out[cu[b]:cu[b + 1]] = (w @ V).view(hkv, n, G, d).permute(1, 0, 2, 3).reshape(n, hq * d)
    return out


def _exact_accept(st):
    cu, par = st["cu"].cpu().numpy(), st["par"].cpu().numpy()
    path = np.full(len(par), -1, np.int32)
    n_path, following = np.zeros(len(cu) - 1, np.int32), np.full(len(cu) - 1, -1, np.int32)
    for b in range(len(cu) - 1):
        c0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        at = 0 if n else None
        while at is not None:
            path[c0 + n_path[b]] = at
            n_path[b] += 1
            following[b] = st["host_sampled"][c0 + at]
            at = next((c for c in range(at + 1, n) if par[c0 + c] == at and st["host_draft"][c0 + c] == following[b]), None)
    return _dev(path), _dev(n_path), _dev(following)


def _exact_commit(st):
    hq, hkv, d, _ = HEADS[st["case"]["heads"]]
    ko, vo = (_dev(a) for a in _slot_index(d))
    cu, seq, table = st["host_cu"], st["host_seq"], st["table"].cpu().numpy()
    path, n_path = st["path"].cpu().numpy(), st["n_path"].cpu().numpy()
    b = np.repeat(np.arange(len(n_path)), n_path)
    i = np.arange(len(b)) - np.repeat(np.cumsum(n_path) - n_path, n_path)
    to = seq[b].astype(np.int64) + i
    at = seq[b].astype(np.int64) + path[cu[b] + i]
    res = []
    for x, off in (("k", ko), ("v", vo)):
        old = st[x].double()
        new = old.clone().view(old.shape[0], old.shape[1], hkv, PAGE * d)
        old = old.view_as(new)
        p_to, p_at = _dev(table[b, to // PAGE].astype(np.int64)), _dev(table[b, at // PAGE].astype(np.int64))
        o_to, o_at = off[_dev(to % PAGE)], off[_dev(at % PAGE)]
        h = torch.arange(hkv, device="cuda").view(1, hkv, 1)
        new[:, p_to[:, None, None], h, o_to[:, None, :]] = old[:, p_at[:, None, None], h, o_at[:, None, :]]
        res.append(new.view(st[x].shape))
    return tuple(res)


def _exact_copy(st):
    res = []
    for x in ("k", "v"):
        old = st[x].double()
        new = old.clone()
        for s, t in zip(st["host_src"].tolist(), st["host_dst"].tolist()):
            new[:, t] = old[:, s]
        res.append(new)
    return tuple(res)
