"""The pages of drafted steps without a GPU: the generator's own bookkeeping over the host allocator, with the layers,
the draws and the commit replaced by stand-ins. A step over trees leaves every sequence with the pages that step()
would have left it with, so that drafts never take a page from a sequence that needs it."""
from collections import namedtuple

import numpy as np
import pytest
import torch

from paper_2608_22167_amd import generate, mcpu, workload as W
from paper_2608_22167_amd.generate import Generator
from tests import tree_reference as R

PAGE = 16
Spec = namedtuple("Spec", "window max_ctx temperature seed n_layers")


def token(sid, pos):
    return 1000 * sid + pos % 7


class Stub(Generator):
    """A generator whose draws are token(sid, pos) and whose pools hold nothing but page ids."""

    def __init__(self, pages_full, pages_sw, window=4096, max_ctx=4096, fail_at=None):
        pool = lambda n: mcpu.KVPool(W.TINY, torch.zeros(n, 1), torch.zeros(n, 1))  # noqa: E731
        self.spec = Spec(window, max_ctx, 0.7, 1, 2)
        self.device, self.max_tokens = "cpu", 256
        self.pools = [pool(pages_sw), pool(pages_full)]
        self.alloc_sw, self.alloc_full = self.pools
        self.seqs, self.held, self.steps = {}, {}, 0
        self.tree_ws = self.ws = self.lm_ws = self.head = None
        self.fail_at, self.calls = fail_at, 0
        self.tree_ws = torch.zeros(256, dtype=torch.uint8)

    def _forward(self, batch, q_lens, tokens, parents=None):
        self.calls += 1
        if self.calls == self.fail_at:
            raise mcpu.McpuError(mcpu.MCPU_EHIP, "a launch failed")
        cu = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        pt_f, pt_s = self._tables(batch, q_lens)
        for b, (s, q) in enumerate(zip(batch, q_lens)):  # every slot that the step writes or sees has a page
            lo, hi = max(0, s.length - self.spec.window + 1) // PAGE, (s.length + q - 1) // PAGE
            assert (pt_f[b, :hi + 1] >= 0).all() and (pt_s[b, lo:hi + 1] >= 0).all()
        x = torch.zeros(len(tokens), 1)
        if parents is None:
            return x, cu
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32))  # noqa: E731
        return x, cu, dict(tok=t(tokens), par=t(parents), sl=None, cu=t(cu), ptf=t(pt_f), pts=t(pt_s))


@pytest.fixture(autouse=True)
def _stand_ins(monkeypatch):
    def sample(head, x, temperature, seed, sids, pos, targets, tok, lp, workspace=None, x_rows=None, **kw):
        for i, (s, p) in enumerate(zip(sids.tolist(), pos.tolist())):
            tok[i] = token(s, p)
        lp.zero_()

    def accept(cu, par, draft, sampled, path, n_path, following, ws):
        for out, got in zip((path, n_path, following), R.accept(*(a.numpy() for a in (cu, par, draft, sampled)))):
            out.copy_(torch.from_numpy(got))

    monkeypatch.setattr(mcpu, "lm_head_sample", sample)
    monkeypatch.setattr(mcpu, "tree_accept", accept)
    monkeypatch.setattr(mcpu, "kv_tree_commit", lambda *a: None)


def state(gen):
    """What every sequence holds: its length, and the logical pages of either kind."""
    return {sid: (s.length, len(s.pages_full), sorted(s.pages_sw)) for sid, s in gen.seqs.items()}


def wrong(n):
    return [-5] * n, [-1] + [0] * (n - 1)


def test_rejected_drafts_leave_the_pages_to_others():
    """Two sequences that fill 6 of 8 pages in 30 steps, with a 63-node draft on the first that is never confirmed."""
    states = []
    for tree in (False, True):
        gen = Stub(8, 8)
        for sid in (0, 1):
            gen.add(sid, range(30))
        gen.step()
        for _ in range(17):
            got = gen.step_tree({0: wrong(63), 1: wrong(3)}) if tree else gen.step()
            assert set(got) == {0, 1}
        states.append((state(gen), gen.free_pages()))
    assert states[0] == states[1]


@pytest.mark.parametrize("window", [20, 4096])
def test_a_tree_step_holds_the_pages_of_plain_steps(window):
    """After every step, confirmed or not: the pages of the tokens fed, and of the window."""
    rng = np.random.default_rng(3)
    plain, gen = Stub(64, 64, window), Stub(64, 64, window)
    for g in (plain, gen):
        for sid, n in ((0, 3), (1, 16), (2, 47)):
            g.add(sid, range(n))
        g.step()
    for _ in range(25):
        drafts = {}
        for sid in (0, 1):
            at = gen.seqs[sid].length + 1  # the position of the token behind the pending one
            run = [token(sid, at + i) for i in range(int(rng.integers(0, 20)))]
            bad, n = int(rng.integers(0, 20)), len(run)
            drafts[sid] = (run[:bad] + [-5] * max(0, n - bad), list(range(-1, n - 1)))
        gen.step_tree(drafts)
        for sid, s in gen.seqs.items():
            while plain.seqs[sid].length < s.length:
                others = {k: plain.seqs.pop(k) for k in list(plain.seqs) if k != sid}
                plain.step()
                plain.seqs.update(others)
        assert state(gen) == state(plain) and gen.free_pages() == plain.free_pages()
    assert max(s.length for s in gen.seqs.values()) > 100


def test_a_held_sequence_keeps_no_page_of_its_drafts():
    gen = Stub(4, 4)
    gen.add(0, range(5))
    gen.step()
    gen.step_tree({0: wrong(40)})
    gen.hold(0)
    gen.add(1, range(48))  # the other three pages
    assert 1 in gen.step()
    assert state(gen) == {0: (6, 1, [0]), 1: (48, 3, [0, 1, 2])}


@pytest.mark.parametrize("pages_full,pages_sw", [(9, 3), (3, 9)])
def test_a_draft_without_room_takes_nothing(pages_full, pages_sw):
    """One kind has pages for the draft, the other has not: neither kind's are kept, within the step or behind it."""
    gen = Stub(pages_full, pages_sw)
    for sid in (0, 1):
        gen.add(sid, range(15))
    gen.step()
    taken = []
    room = gen._room
    gen._room = lambda s, q: (room(s, q), taken.append(gen.free_pages()))[0]
    got = gen.step_tree({0: wrong(40), 1: ([token(1, 16)], [-1])})
    # the first one's draft has no room and gives its pages back before the second one's is tried
    assert [len(got[sid]) for sid in (0, 1)] == [1, 2] and taken[0] == (pages_full - 2, pages_sw - 2)
    assert state(gen) == {0: (16, 1, [0]), 1: (17, 2, [0, 1])}


def test_a_step_that_fails_gives_its_draft_pages_back():
    gen = Stub(8, 8, fail_at=2)
    gen.add(0, range(10))
    gen.step()
    before = state(gen), gen.free_pages()
    with pytest.raises(mcpu.McpuError):
        gen.step_tree({0: wrong(50)})
    assert (state(gen), gen.free_pages()) == before
    assert gen.step_tree({0: ([token(0, 11)], [-1])})[0] == [(token(0, 11), 0.0), (token(0, 12), 0.0)]


@pytest.mark.parametrize("error", [mcpu.McpuError(mcpu.MCPU_EHIP, "a launch failed"), RuntimeError("out of memory")])
@pytest.mark.parametrize("fail_at", [1, 2])
def test_a_fork_that_fails_leaves_every_page_as_it_was(monkeypatch, error, fail_at):
    """The copy of the last page fails for the first or the second kind: no page is shared, taken or forgotten."""
    gen = Stub(32, 32)
    gen.add(0, range(40))
    gen.step()
    holders = lambda: [mcpu.kv_page_holders(p, i) for p in gen.pools for i in range(32)]  # noqa: E731
    before = state(gen), gen.free_pages(), holders()
    calls = []

    def copy(*a):
        calls.append(a)
        if len(calls) == fail_at:
            raise error

    monkeypatch.setattr(mcpu, "kv_pages_copy", copy)
    with pytest.raises(type(error)):
        gen.fork(0, [1, 2, 3])
    assert len(calls) == fail_at and (state(gen), gen.free_pages(), holders()) == before
    gen.fork(0, [1, 2, 3])
    assert state(gen) == {sid: (40, 3, [0, 1, 2]) for sid in range(4)}
    for sid in range(4):
        gen.release(sid)
    assert gen.free_pages() == (32, 32)


def test_a_group_that_fails_leaves_no_sequence(monkeypatch):
    gen = Stub(32, 32)

    def copy(*a):
        raise RuntimeError("out of memory")

    monkeypatch.setattr(mcpu, "kv_pages_copy", copy)
    with pytest.raises(RuntimeError):
        gen.add_group([4, 5], range(40))
    assert not gen.seqs and gen.free_pages() == (32, 32)
