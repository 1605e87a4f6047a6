"""Continuous-batching generation over the decoder stack (argument
marshalling and host bookkeeping around the C ABI; every step of the model
runs in libmcpu.so's kernels).

The Run stage of the paper's rollout pipeline keeps many multi-turn
trajectories in flight on one policy replica: each turn the policy generates
tokens at the rollout temperature, the trajectory then waits on a tool, and
the tool's observation joins the context before the next turn (Sec. 1 and
Sec. 3.2; temperature 0.7 in the training-details appendix). `Generator`
serves that pattern. Every call to `step()` advances all sequences that have
input: a prompt or observation chunk is prefilled (chunked prefill through
the same decode_layer call), a decoding sequence feeds its last sampled token,
and every sequence that reached the end of its input samples one new token.

Pages are allocated per step as sequences grow (kv_pages_alloc, one pool id
space per attention kind: the same page ids index every layer of that kind),
pages of sliding-window layers are freed once they fall wholly left of the
window, and all of a sequence's pages are freed when it is released.
`score()` recomputes the log-probabilities of whole trajectories (the GRPO
update's log-prob pass): a long causal prefill with targets, no sampling.

`add_group()` starts the members of a group (the policy update compares several
trajectories of one prompt) on pages that they share: the prompt is prefilled
once, `fork()` gives every member the whole pages and a copy of the last, partly
filled one. `step_tree()` verifies drafted tokens: where a drafted token equals the
draw before it, the step yields more than one token per sequence, and because a
draw depends only on (seed, sequence, position) they are the tokens that `step()`
would have drawn one by one, but where two ids nearly tie: steps of other row counts
round differently. `Lookup` drafts from the sequence's own history.
"""
from __future__ import annotations

from collections import deque
from dataclasses import dataclass, field
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

from paper_2608_22167_amd import mcpu, workload as W

PAGE = 16


@dataclass
class GenSpec:
    """A decoder stack with its generation ends. Layer i uses the window if i
    is even (0-based) and full attention if odd, like the 24-layer stack."""
    n_layers: int
    base: W.LayerShape            # bf16 layer shape (experts MXFP4)
    vocab: int
    seed: int = 3001
    window: int = 128
    pages_full: int = 4096        # pages per full-attention layer pool
    pages_sw: int = 1024          # pages per sliding-window layer pool
    max_ctx: int = 65536          # positions the RoPE table covers
    temperature: float = float(np.float32(0.7))

    def stack_spec(self) -> W.StackSpec:
        full = W.replace(self.base, expert_fmt="mxfp4", window=0)
        sw = W.replace(full, window=self.window)
        z = np.zeros((0, 1), np.int32)
        return W.StackSpec(name="generator", seed=self.seed, n_layers=self.n_layers, shape_full=full, shape_sw=sw,
                           seq_lens=np.zeros(0, np.int32), page_table_full=z, n_pages_full=self.pages_full,
                           page_table_sw=z, n_pages_sw=self.pages_sw, rope_max_pos=self.max_ctx)


@dataclass
class _Seq:
    sid: int
    length: int = 0                                     # tokens in the cache
    pending: List[int] = field(default_factory=list)    # input not yet fed
    pages_full: List[int] = field(default_factory=list)  # logical page i -> physical id
    pages_sw: Dict[int, int] = field(default_factory=dict)
    history: List[int] = field(default_factory=list)    # every token fed so far


class Lookup:
    """Drafts from one sequence's own tokens: what followed the latest places at
    which its last tokens stood before (the last `ngram`, of fewer where there is
    no such place). Tool observations and the model's quotes of them repeat."""

    def __init__(self, ngram: int = 3, width: int = 2):
        self.ngram, self.width = ngram, width
        self.after: Dict[tuple, deque] = {}   # tokens -> the latest positions behind them
        self.history: List[int] = []

    def feed(self, tokens: Sequence[int]) -> None:
        """The tokens that follow those fed so far."""
        h = self.history
        for t in tokens:
            i = len(h)
            for n in range(1, min(self.ngram, i) + 1):
                self.after.setdefault(tuple(h[i - n:i]), deque(maxlen=self.width)).append(i)
            h.append(t)

    def tree(self, history: Sequence[int], max_nodes: int, max_depth: int) -> Tuple[List[int], List[int]]:
        """`draft` behind `history`, a longer one than was fed so far, with the same
        beginning."""
        self.feed(history[len(self.history):])
        return self.draft(max_nodes, max_depth)

    def draft(self, max_nodes: int, max_depth: int) -> Tuple[List[int], List[int]]:
        """At most max_nodes tokens, max_depth in a row, to follow the tokens fed; the
        places' common beginnings are shared. Returns the tokens and their parents
        (index of the token before, -1: the last one fed)."""
        history = self.history
        places: Sequence[int] = ()
        for n in range(min(self.ngram, len(history)), 0, -1):
            places = self.after.get(tuple(history[-n:]), ())
            if places:
                break
        runs = [history[p:p + max_depth] for p in reversed(places)]
        tokens: List[int] = []
        parents: List[int] = []
        child: Dict[Tuple[int, int], int] = {}
        ends = [-1] * len(runs)
        for d in range(max_depth):        # level by level, so that a cut at max_nodes keeps every branch
            for r, run in enumerate(runs):
                if d >= len(run) or (d and ends[r] < 0):
                    continue
                key = (ends[r], run[d])
                if key not in child:
                    if len(tokens) >= max_nodes:
                        return tokens, parents
                    child[key] = len(tokens)
                    tokens.append(run[d])
                    parents.append(ends[r])
                ends[r] = child[key]
        return tokens, parents


class Generator:
    """The stack's weights, one K/V pool pair per layer, the embedding and the
    vocabulary head, all resident on the GPU; sequences come and go."""

    def __init__(self, spec: GenSpec, device="cuda", max_tokens_per_step: int = 8192):
        self.spec = spec
        self.ss = ss = spec.stack_spec()
        self.device = device
        self.weights, self.k, self.v, self.pools = [], [], [], []
        for i in range(spec.n_layers):
            s = ss.shape(i)
            self.weights.append(mcpu.DeviceWeights(s, W.stack_weights_device(ss, i, device), device))
            n = ss.n_pages(i)
            self.k.append(torch.zeros((n, s.n_kv_heads, PAGE, s.head_dim), dtype=torch.bfloat16, device=device))
            self.v.append(torch.zeros_like(self.k[-1]))
            self.pools.append(mcpu.KVPool(s, self.k[-1], self.v[-1]))
        # page ids are handed out by the first pool of each kind and used in every layer of that kind
        self.alloc_full = self.pools[1] if spec.n_layers > 1 else None
        self.alloc_sw = self.pools[0]
        lm = W.lm_weights_device(spec.seed, ss.shape_full.hidden, spec.vocab, device)
        self.tree_ws = None  # workspace of step_tree, made at its first call
        self.embed = lm["embed"]
        self.head = mcpu.DeviceLmHead(lm["g_final"], lm["w_lm"], ss.shape_full.rms_eps, device)
        self.max_tokens = max_tokens_per_step
        s0 = ss.shape_full
        self.ws = mcpu.workspace(max(mcpu.decode_layer_workspace_size(ss.shape(i), max_tokens_per_step,
                                                                      max_tokens_per_step)
                                     for i in range(min(2, spec.n_layers))), device)
        self.lm_ws = mcpu.workspace(mcpu.lm_head_workspace_size(s0.hidden, spec.vocab, max_tokens_per_step), device)
        self.seqs: Dict[int, _Seq] = {}
        self.held: Dict[int, List[int]] = {}   # a sequence's sampled token kept back while its turn waits
        self.steps = 0

    # ------------------------------------------------------------------ sequences

    def add(self, sid: int, tokens: Sequence[int]) -> None:
        """Queue input for sequence sid (a new trajectory's prompt, or a tool
        observation appended to a waiting one)."""
        if not len(tokens):
            return
        s = self.seqs.setdefault(sid, _Seq(sid))
        s.pending.extend(int(t) for t in tokens)

    def release(self, sid: int) -> None:
        """Free every page of sequence sid and forget it."""
        s = self.seqs.pop(sid)
        self.held.pop(sid, None)
        if self.alloc_full is not None and s.pages_full:
            mcpu.kv_pages_free(self.alloc_full, np.array(s.pages_full, np.int32))
        if s.pages_sw:
            mcpu.kv_pages_free(self.alloc_sw, np.array(list(s.pages_sw.values()), np.int32))

    def fork(self, sid: int, new_sids: Sequence[int]) -> None:
        """Start each of new_sids as a copy of sequence sid (cache, history and
        pending input): whole pages get another holder, a partly filled last
        page is copied for each. All or nothing: a fork that fails (MCPU_ENOMEM:
        too few pages) leaves every sequence and page as it was."""
        s, n = self.seqs[sid], len(new_sids)
        if len(set(new_sids)) != n or any(k in self.seqs for k in new_sids):
            raise ValueError(f"fork: sequence ids {list(new_sids)} repeat or exist")
        if n == 0:
            return
        whole, part = s.length // PAGE, s.length % PAGE > 0
        kinds = []  # (allocator, layer pools, shared pages, last page, its copies)
        for alloc, pools, shared, last in (
                (self.alloc_full, self.pools[1::2], s.pages_full[:whole], s.pages_full[whole:whole + 1]),
                (self.alloc_sw, self.pools[0::2], [p for lp, p in s.pages_sw.items() if lp < whole],
                 [p for lp, p in s.pages_sw.items() if lp == whole])):
            if alloc is not None:
                kinds.append((alloc, pools, shared, last if part else []))
        copies: List[np.ndarray] = []
        taken: List[tuple] = []  # (allocator, pages), a holder each
        try:
            for alloc, _, shared, last in kinds:
                copies.append(mcpu.kv_pages_alloc(alloc, n * len(last)))
                taken.append((alloc, copies[-1]))
                for _ in range(n):
                    mcpu.kv_pages_share(alloc, shared)
                    taken.append((alloc, shared))
            for (_, pools, _, last), ids in zip(kinds, copies):
                if not last:
                    continue
                src = np.full(n, last[0], np.int32)
                d_src, d_dst = (torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(self.device) for a in (src, ids))
                for i in range(0, len(pools), mcpu.MAX_POOLS):
                    mcpu.kv_pages_copy(pools[i:i + mcpu.MAX_POOLS], d_src, d_dst, src, ids, self.ws)
        except BaseException:
            for alloc, ids in taken:
                mcpu.kv_pages_free(alloc, ids)
            raise
        full = copies[0] if self.alloc_full is not None else np.zeros(0, np.int32)
        for j, k in enumerate(new_sids):
            c = _Seq(k, s.length, list(s.pending), s.pages_full[:whole], {}, list(s.history))
            if part and self.alloc_full is not None:
                c.pages_full.append(int(full[j]))
            c.pages_sw = {lp: p for lp, p in s.pages_sw.items() if lp < whole}
            if part and len(copies[-1]):
                c.pages_sw[whole] = int(copies[-1][j])
            self.seqs[k] = c
            if sid in self.held:
                self.held[k] = list(self.held[sid])

    def add_group(self, sids: Sequence[int], tokens: Sequence[int]) -> None:
        """Start the sequences sids on one prompt: its tokens but the last are
        prefilled once and shared, the last is each member's pending input, so
        that every member draws its own next token."""
        tokens = [int(t) for t in tokens]
        if not len(sids) or not tokens:
            raise ValueError("add_group needs sequence ids and a prompt")
        if len(set(sids)) != len(sids) or any(k in self.seqs for k in sids):
            raise ValueError(f"add_group: sequence ids {list(sids)} repeat or exist")
        s = self.seqs[sids[0]] = _Seq(sids[0], pending=tokens)
        try:
            while len(s.pending) > 1:
                q = min(len(s.pending) - 1, self.max_tokens)
                self._grow(s, q)
                self._forward([s], [q], np.array(s.pending[:q], np.int64))
                s.history.extend(s.pending[:q])
                del s.pending[:q]
                s.length += q
                self._shrink(s)
            self.fork(sids[0], sids[1:])
        except BaseException:
            self.release(sids[0])
            raise

    def free_pages(self):
        return (self.alloc_full.free_pages() if self.alloc_full is not None else 0, self.alloc_sw.free_pages())

    def _grow(self, s: _Seq, q: int) -> None:
        """Pages for positions s.length .. s.length + q - 1: every full-layer
        page up to the last, and every window page the new tokens can see."""
        last = s.length + q - 1
        if self.alloc_full is not None:
            need = last // PAGE + 1 - len(s.pages_full)
            if need > 0:
                s.pages_full.extend(int(p) for p in mcpu.kv_pages_alloc(self.alloc_full, need))
        lo = max(0, s.length - self.spec.window + 1) // PAGE
        missing = [lp for lp in range(lo, last // PAGE + 1) if lp not in s.pages_sw]
        if missing:
            for lp, p in zip(missing, mcpu.kv_pages_alloc(self.alloc_sw, len(missing))):
                s.pages_sw[lp] = int(p)

    def _room(self, s: _Seq, q: int) -> bool:
        """_grow, or False where there are too few pages (only the pending token's stay with the sequence)."""
        try:
            self._grow(s, q)
        except mcpu.McpuError as e:
            if e.code != mcpu.MCPU_ENOMEM:
                raise
            self._trim([s], 1)
            return False
        return True

    def _trim(self, seqs: Sequence[_Seq], more: int = 0) -> None:
        """Free the pages behind position s.length + more - 1 of each sequence, which drafted tokens that did not
        stay have taken. One call for each kind: sequence by sequence a step of 48 trees took 0.15-0.2 ms more."""
        full: List[int] = []
        window: List[int] = []
        for s in seqs:
            keep = (s.length + more + PAGE - 1) // PAGE
            full += s.pages_full[keep:]
            del s.pages_full[keep:]
            window += [s.pages_sw.pop(lp) for lp in [lp for lp in s.pages_sw if lp >= keep]]
        for alloc, pages in ((self.alloc_full, full), (self.alloc_sw, window)):
            if pages:
                mcpu.kv_pages_free(alloc, np.array(pages, np.int32))

    def _shrink(self, s: _Seq) -> None:
        """Free window pages wholly left of the next token's window."""
        lo = max(0, s.length - self.spec.window + 1) // PAGE
        old = [lp for lp in s.pages_sw if lp < lo]
        if old:
            mcpu.kv_pages_free(self.alloc_sw, np.array([s.pages_sw.pop(lp) for lp in old], np.int32))

    # ------------------------------------------------------------------ one step

    def _tables(self, batch: List[_Seq], q_lens: List[int]):
        max_lp = max((s.length + q - 1) // PAGE + 1 for s, q in zip(batch, q_lens))
        pt_f = -np.ones((len(batch), max_lp), np.int32)
        pt_s = -np.ones((len(batch), max_lp), np.int32)
        for b, s in enumerate(batch):
            own = s.pages_full[:max_lp]  # a step that failed may have left pages behind the last position
            pt_f[b, :len(own)] = own
            for lp, p in s.pages_sw.items():
                if lp < max_lp:
                    pt_s[b, lp] = p
        return pt_f, pt_s

    def _forward(self, batch: List[_Seq], q_lens: List[int], tokens: np.ndarray, parents: Optional[np.ndarray] = None):
        """Embeds the step's input tokens and runs every layer; returns the
        final residual rows [T, H] and cu_q. With parents, the input of each
        sequence is a tree of tokens, whose accepted path is still to be kept
        (the device arrays for that are returned too)."""
        T = int(sum(q_lens))
        dev = self.device
        cu = np.zeros(len(batch) + 1, np.int32)
        cu[1:] = np.cumsum(q_lens)
        seq_lens = np.array([s.length for s in batch], np.int32)
        pt_f, pt_s = self._tables(batch, q_lens)
        d_tok = torch.from_numpy(tokens.astype(np.int32)).to(dev)
        d_sl = torch.from_numpy(seq_lens).to(dev)
        d_cu = torch.from_numpy(cu).to(dev)
        d_ptf, d_pts = torch.from_numpy(pt_f).to(dev), torch.from_numpy(pt_s).to(dev)
        H = self.ss.shape_full.hidden
        x = [torch.empty((T, H), device=dev), torch.empty((T, H), device=dev)]
        mcpu.embed_tokens(self.embed, d_tok, x[0], self.ws)
        d_par = None if parents is None else torch.from_numpy(parents).to(dev)
        for i in range(self.spec.n_layers):
            table = d_pts if self.ss.is_sw(i) else d_ptf
            if parents is None:
                mcpu.decode_layer(self.ss.shape(i), self.weights[i], self.pools[i], table, d_sl, d_cu, seq_lens, cu,
                                  x[i % 2], x[(i + 1) % 2], workspace=self.ws)
            else:
                mcpu.decode_layer_tree(self.ss.shape(i), self.weights[i], self.pools[i], table, d_sl, d_cu, d_par,
                                       seq_lens, cu, x[i % 2], x[(i + 1) % 2], workspace=self.tree_ws)
        out = x[self.spec.n_layers % 2]
        return (out, cu) if parents is None else (out, cu, dict(tok=d_tok, par=d_par, sl=d_sl, cu=d_cu, ptf=d_ptf, pts=d_pts))

    def step(self) -> Dict[int, tuple]:
        """Advance every sequence with pending input by up to its whole input
        (bounded by max_tokens_per_step in total, oldest first). Returns
        {sid: (token, logprob)} for the sequences that sampled a token; a
        sampled token becomes that sequence's next input unless the caller
        calls `hold(sid)` (e.g. a tool call ends the turn)."""
        ready = [s for s in self.seqs.values() if s.pending]
        batch, q_lens, budget = [], [], self.max_tokens
        for s in ready:
            if budget <= 0:
                break
            q = min(len(s.pending), budget)
            batch.append(s)
            q_lens.append(q)
            budget -= q
        if not batch:
            return {}
        for s, q in zip(batch, q_lens):
            self._grow(s, q)
        tokens = np.concatenate([np.array(s.pending[:q], np.int64) for s, q in zip(batch, q_lens)])
        x, cu = self._forward(batch, q_lens, tokens)
        # sample for the sequences whose whole input has been fed
        done = [b for b, (s, q) in enumerate(zip(batch, q_lens)) if q == len(s.pending)]
        out = {}
        if done:
            dev = self.device
            rows = torch.from_numpy(np.array([cu[b + 1] - 1 for b in done], np.int32)).to(dev)
            sids = torch.from_numpy(np.array([batch[b].sid for b in done], np.int32)).to(dev)
            pos = torch.from_numpy(np.array([batch[b].length + q_lens[b] for b in done], np.int32)).to(dev)
            n = len(done)
            tok = torch.empty(n, dtype=torch.int32, device=dev)
            lp = torch.empty(n, device=dev)
            mcpu.lm_head_sample(self.head, x, self.spec.temperature, self.spec.seed, sids, pos, None, tok, lp,
                                workspace=self.lm_ws, x_rows=rows)
            tok_h, lp_h = tok.cpu().numpy(), lp.cpu().numpy()
            for j, b in enumerate(done):
                out[batch[b].sid] = (int(tok_h[j]), float(lp_h[j]))
        for b, (s, q) in enumerate(zip(batch, q_lens)):
            s.history.extend(s.pending[:q])
            del s.pending[:q]
            s.length += q
            self._shrink(s)
            if s.sid in out:
                s.pending.append(out[s.sid][0])
        self.steps += 1
        return out

    def step_tree(self, drafts: Dict[int, Tuple[Sequence[int], Sequence[int]]]) -> Dict[int, List[tuple]]:
        """Advance every decoding sequence (one pending token) with a tree of
        drafted tokens behind it: drafts[sid] = (tokens, parents), parents being
        indices into tokens or -1 for the pending token; at most
        TREE_MAX_NODES - 1 of them, none for a sequence without a draft.
        Returns {sid: [(token, logprob), ...]}: the draws along the confirmed
        path, one at least, of which the last becomes the pending token. They
        are the tokens that calls of `step()` would have drawn, outside near ties
        (the scores of two ids within the rounding of a step). Sequences with
        longer input are left to `step()`; no more rows are fed than
        max_tokens_per_step, oldest sequences first and drafts only where every
        sequence has its row. A draft for which there are no rows or pages left, or
        that passes the last position, is not tried. Pages of tokens that did not
        stay are free again when the call returns or fails, so that a sequence
        holds what `step()` would have left it with."""
        trees = []
        for s in [s for s in self.seqs.values() if len(s.pending) == 1][:self.max_tokens]:
            d_tok, d_par = drafts.get(s.sid, ((), ()))
            if len(d_tok) != len(d_par) or len(d_tok) >= mcpu.TREE_MAX_NODES:
                raise ValueError(f"draft of sequence {s.sid}: {len(d_tok)} tokens, {len(d_par)} parents")
            dep = [0]
            for i, p in enumerate(d_par):
                if not -1 <= p < i:
                    raise ValueError(f"draft of sequence {s.sid}: parent {p} of token {i}")
                dep.append(dep[p + 1] + 1)
            trees.append((s, d_tok, d_par, dep))
        try:
            return self._step_trees(trees)
        finally:
            self._trim([s for s, *_ in trees])

    def _step_trees(self, trees) -> Dict[int, List[tuple]]:
        """step_tree of checked drafts: (sequence, tokens, parents, depths from the pending token on)."""
        batch, q_lens, toks, pars, depth, budget = [], [], [], [], [], self.max_tokens - len(trees)
        for s, *_ in trees:
            self._grow(s, 1)
        for s, d_tok, d_par, dep in trees:
            if len(d_tok) > budget or s.length + max(dep) >= self.spec.max_ctx or not self._room(s, 1 + len(d_tok)):
                d_tok, d_par, dep = (), (), [0]
            budget -= len(d_tok)
            batch.append(s)
            q_lens.append(1 + len(d_tok))
            toks += [s.pending[0], *(int(t) for t in d_tok)]
            pars += [-1, *(int(p) + 1 for p in d_par)]
            depth += dep
        if not batch:
            return {}
        if self.tree_ws is None:
            self.tree_ws = mcpu.workspace(max(mcpu.decode_layer_tree_workspace_size(self.ss.shape(i), self.max_tokens,
                                                                                    self.max_tokens)
                                              for i in range(min(2, self.spec.n_layers))), self.device)
        x, cu, d = self._forward(batch, q_lens, np.array(toks, np.int64), np.array(pars, np.int32))
        dev, T, B = self.device, len(toks), len(batch)
        up = lambda a: torch.from_numpy(np.array(a, np.int32)).to(dev)  # noqa: E731
        lens = np.repeat([s.length for s in batch], q_lens)
        sampled = torch.empty(T, dtype=torch.int32, device=dev)
        lp = torch.empty(T, device=dev)
        mcpu.lm_head_sample(self.head, x, self.spec.temperature, self.spec.seed,
                            up(np.repeat([s.sid for s in batch], q_lens)), up(lens + np.array(depth) + 1), None, sampled,
                            lp, workspace=self.lm_ws)
        path, n_path, following = (torch.empty(n, dtype=torch.int32, device=dev) for n in (T, B, B))
        mcpu.tree_accept(d["cu"], d["par"], d["tok"], sampled, path, n_path, following, self.tree_ws)
        for pools, table in ((self.pools[0::2], d["pts"]), (self.pools[1::2], d["ptf"])):
            for i in range(0, len(pools), mcpu.MAX_POOLS):
                mcpu.kv_tree_commit(pools[i:i + mcpu.MAX_POOLS], table, d["sl"], d["cu"], path, n_path, self.tree_ws)
        path, n_path, sampled, lp = path.cpu().numpy(), n_path.cpu().numpy(), sampled.cpu().numpy(), lp.cpu().numpy()
        out = {}
        for b, s in enumerate(batch):
            rows = cu[b] + path[cu[b]:cu[b] + n_path[b]]
            out[s.sid] = [(int(sampled[r]), float(lp[r])) for r in rows]
            s.history.extend(int(toks[r]) for r in rows)
            s.length += len(rows)
            s.pending = [int(sampled[rows[-1]])]
            self._shrink(s)
        self.steps += 1
        return out

    def hold(self, sid: int) -> None:
        """Drop the sequence's pending sampled token (its turn ended); the
        token is still part of the trajectory: it is fed with the next input."""
        s = self.seqs[sid]
        self.held[sid] = s.pending[:]
        s.pending.clear()

    def resume(self, sid: int, observation: Sequence[int]) -> None:
        """Append a tool observation after the held token."""
        held = self.held.pop(sid, [])
        self.add(sid, list(held) + list(observation))

    def check_errors(self) -> int:
        bits = mcpu.mcpu_check_device_errors(self.ws) | mcpu.mcpu_check_device_errors(self.lm_ws)
        return bits | (mcpu.mcpu_check_device_errors(self.tree_ws) if self.tree_ws is not None else 0)

    # ------------------------------------------------------------------ trajectory scoring

    def score(self, trajectories: Sequence[Sequence[int]], sid_base: int = 1 << 20,
              temperature: Optional[float] = None) -> List[np.ndarray]:
        """Log-probability of every token of each trajectory given its prefix
        (token 0 has none), under softmax(logits / temperature): the whole
        trajectories are prefilled in chunks of at most max_tokens_per_step
        tokens in all, with the next tokens as targets. Pages are taken from
        and returned to the pools."""
        tau = self.spec.temperature if temperature is None else temperature
        trajectories = [np.asarray(t, np.int64) for t in trajectories]
        res = [np.zeros(max(len(t) - 1, 0), np.float64) for t in trajectories]
        states = [_Seq(sid_base + i) for i in range(len(trajectories))]
        try:
            while True:
                batch, q_lens, idx, budget = [], [], [], self.max_tokens
                for i, (s, tr) in enumerate(zip(states, trajectories)):
                    left = len(tr) - s.length
                    if left > 0 and budget > 0:
                        q = min(left, budget)
                        batch.append(s)
                        q_lens.append(q)
                        idx.append(i)
                        budget -= q
                if not batch:
                    break
                for s, q in zip(batch, q_lens):
                    self._grow(s, q)
                tokens = np.concatenate([trajectories[i][s.length:s.length + q]
                                         for i, s, q in zip(idx, batch, q_lens)])
                x, cu = self._forward(batch, q_lens, tokens)
                # targets: the token after each row (the last row of a trajectory has none)
                rows, tgts, spans = [], [], []
                for b, (i, s, q) in enumerate(zip(idx, batch, q_lens)):
                    n_t = min(q, len(trajectories[i]) - 1 - s.length)
                    if n_t > 0:
                        rows.append(cu[b] + np.arange(n_t, dtype=np.int32))
                        tgts.append(trajectories[i][s.length + 1:s.length + 1 + n_t])
                        spans.append((i, s.length, n_t))
                if rows:
                    dev = self.device
                    rows, tgts = np.concatenate(rows), np.concatenate(tgts).astype(np.int32)
                    tlp = torch.empty(len(rows), device=dev)
                    mcpu.lm_head_sample(self.head, x, tau, 0, None, None, torch.from_numpy(tgts).to(dev), None, None,
                                        tlp, workspace=self.lm_ws, x_rows=torch.from_numpy(rows).to(dev))
                    vals = tlp.cpu().numpy()
                    at = 0
                    for i, p, n_t in spans:
                        res[i][p:p + n_t] = vals[at:at + n_t]
                        at += n_t
                for s, q in zip(batch, q_lens):
                    s.length += q
                    self._shrink(s)
        finally:
            for s in states:
                if self.alloc_full is not None and s.pages_full:
                    mcpu.kv_pages_free(self.alloc_full, np.array(s.pages_full, np.int32))
                if s.pages_sw:
                    mcpu.kv_pages_free(self.alloc_sw, np.array(list(s.pages_sw.values()), np.int32))
        return res
