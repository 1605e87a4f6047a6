"""Trees of drafted tokens and shared pages without a GPU: refusals (every call
returns on the host; addresses are dummies that nothing reads) and page holders."""
import ctypes
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2608_22167_amd import mcpu, workload as W
from tests import tree_reference as R

D = 1 << 32  # a dummy device address


def _pool(shape=W.TINY, n_pages=64, k=4096, v=8192):
    h = ctypes.c_void_p()
    assert mcpu.lib().kv_pool_create(ctypes.byref(mcpu.make_cfg(shape)), n_pages, k, v, ctypes.byref(h)) == 0
    return h


def _i32(*a):
    return np.array(a, np.int32)


def _error():
    return mcpu.lib().mcpu_last_error().decode()


def _attention(shape=W.TINY, pool=None, seq=(5, 17), cu=(0, 3, 4), max_pages=8, ws=None, batch=2, **null):
    a = dict(table=D, seq_lens=D, cu_q=D, parents=D, q=D, o=D, workspace=D)
    a.update({k: v for k, v in null.items()})
    hs, hc = _i32(*seq), _i32(*cu)
    cfg = mcpu.make_cfg(shape)
    need = mcpu.tree_attention_workspace_size(shape, batch, cu[-1]) if ws is None else ws
    return mcpu.lib().tree_attention(ctypes.byref(cfg), None, pool or _pool(shape), batch, a["table"], max_pages,
                                     a["seq_lens"], a["cu_q"], a["parents"], a.get("hs", hs.ctypes.data),
                                     a.get("hc", hc.ctypes.data), a["q"], a["o"], a["workspace"], need, None)


def test_attention_refusals():
    for name in ("table", "seq_lens", "cu_q", "parents", "q", "o", "workspace", "hs", "hc"):
        assert _attention(**{name: None}) == mcpu.MCPU_EINVAL, name
        assert "NULL" in _error()
    assert _attention(batch=0) == mcpu.MCPU_EINVAL
    assert _attention(max_pages=0) == mcpu.MCPU_EINVAL
    assert _attention(cu=(1, 3, 4)) == mcpu.MCPU_EINVAL
    assert _attention(cu=(0, 3, 2)) == mcpu.MCPU_EINVAL
    assert _attention(seq=(-1, 4)) == mcpu.MCPU_EINVAL
    assert _attention(cu=(0, 65, 66)) == mcpu.MCPU_EUNSUPPORTED and "65 nodes" in _error()
    assert _attention(seq=(5, 8 * 16)) == mcpu.MCPU_EINVAL and "beyond page table" in _error()
    assert _attention(seq=(2 ** 31 - 1, 4)) == mcpu.MCPU_EINVAL and "beyond page table" in _error()
    assert _attention(q=D + 8) == mcpu.MCPU_EINVAL and "aligned" in _error()
    assert _attention(pool=_pool(replace(W.TINY, head_dim=64))) == mcpu.MCPU_EINVAL
    need = mcpu.tree_attention_workspace_size(W.TINY, 2, 4)
    assert _attention(ws=need - 256) == mcpu.MCPU_ENOMEM
    assert _attention(cu=(0, 0, 0)) == mcpu.MCPU_OK  # no node: nothing is launched
    assert mcpu.tree_attention_workspace_size(replace(W.TINY, page_size=8), 2, 4) == 0
    assert mcpu.tree_attention_workspace_size(W.TINY, -1, 4) == 0


def test_accept_refusals():
    L = mcpu.lib()
    a = [D] * 8

    def call(batch=2, n=4, ws=256, drop=None):
        p = list(a)
        if drop is not None:
            p[drop] = None
        return L.tree_accept(batch, n, *p, ws, None)

    for i in range(8):
        assert call(drop=i) == mcpu.MCPU_EINVAL, i
    assert call(batch=-1) == mcpu.MCPU_EINVAL and call(n=-1) == mcpu.MCPU_EINVAL
    assert call(ws=255) == mcpu.MCPU_ENOMEM
    assert call(batch=0) == mcpu.MCPU_OK


def _handles(*pools):
    return (ctypes.c_void_p * len(pools))(*pools)


def test_commit_refusals():
    L = mcpu.lib()
    p, other = _pool(), _pool(k=1 << 20, v=2 << 20)

    def call(pools=_handles(p, other), n_pools=2, batch=2, max_pages=8, n=4, ws=256, drop=None):
        q = [D] * 6
        if drop is not None:
            q[drop] = None
        return L.kv_tree_commit(pools, n_pools, batch, q[0], max_pages, q[1], q[2], n, q[3], q[4], q[5], ws, None)

    for i in range(6):
        assert call(drop=i) == mcpu.MCPU_EINVAL, i
    assert call(pools=None) == mcpu.MCPU_EINVAL
    assert call(n_pools=0) == mcpu.MCPU_EINVAL
    assert call(n_pools=65) == mcpu.MCPU_EUNSUPPORTED
    assert call(pools=_handles(p, p)) == mcpu.MCPU_EINVAL and "the same" in _error()
    assert call(pools=_handles(p, _pool(k=4096, v=2 << 20))) == mcpu.MCPU_EINVAL
    assert call(pools=_handles(p, None)) == mcpu.MCPU_EINVAL
    assert call(pools=_handles(p, _pool(replace(W.TINY, n_kv_heads=4), k=1 << 20, v=2 << 20))) == mcpu.MCPU_EINVAL
    assert call(batch=-1) == mcpu.MCPU_EINVAL and call(n=-1) == mcpu.MCPU_EINVAL and call(max_pages=0) == mcpu.MCPU_EINVAL
    assert call(ws=255) == mcpu.MCPU_ENOMEM
    assert call(batch=0) == mcpu.MCPU_OK and call(n=0) == mcpu.MCPU_OK


def test_copy_refusals():
    L = mcpu.lib()
    p, small = _pool(), _pool(n_pages=10, k=1 << 20, v=2 << 20)

    def call(src, dst, pools=_handles(p), n=None, src_d=D, dst_d=D, ws_d=D, ws=256, host=True):
        s, d = _i32(*src), _i32(*dst)
        return L.kv_pages_copy(pools, len(pools), len(s) if n is None else n, src_d, dst_d,
                               s.ctypes.data if host else None, d.ctypes.data, ws_d, ws, None)

    assert call([], []) == mcpu.MCPU_OK
    assert call([1], [2], n=-1) == mcpu.MCPU_EINVAL
    for kw in (dict(src_d=None), dict(dst_d=None), dict(ws_d=None), dict(host=False)):
        assert call([1], [2], **kw) == mcpu.MCPU_EINVAL
    assert call([1], [2], ws=128) == mcpu.MCPU_ENOMEM
    for s, d in (([1], [64]), ([64], [1]), ([-1], [1]), ([1], [-1])):
        assert call(s, d) == mcpu.MCPU_EINVAL and "outside" in _error()
    assert call([1], [10], pools=_handles(p, small)) == mcpu.MCPU_EINVAL  # beyond the smaller pool
    assert call([1, 2], [5, 5]) == mcpu.MCPU_EINVAL and "repeated" in _error()
    assert call([1, 2], [2, 3]) == mcpu.MCPU_EINVAL and "source and a destination" in _error()
    assert call([7], [7]) == mcpu.MCPU_EINVAL


def test_page_holders():
    L = mcpu.lib()
    p = _pool(n_pages=6)
    ids = np.zeros(4, np.int32)
    assert L.kv_pages_alloc(p, 4, ids.ctypes.data) == 0
    holders = lambda: [L.kv_page_holders(p, i) for i in range(6)]  # noqa: E731
    assert holders() == [1, 1, 1, 1, 0, 0]
    again = _i32(0, 1, 1)
    assert L.kv_pages_share(p, 3, again.ctypes.data) == 0
    assert holders() == [2, 3, 1, 1, 0, 0] and L.kv_pool_free_pages(p) == 2
    for bad in (_i32(0, 4), _i32(0, 6), _i32(-1, 0)):  # free, out of range: nothing is added
        assert L.kv_pages_share(p, 2, bad.ctypes.data) == mcpu.MCPU_EINVAL
    assert holders() == [2, 3, 1, 1, 0, 0]
    assert L.kv_pages_share(None, 1, again.ctypes.data) == mcpu.MCPU_EINVAL
    assert L.kv_pages_share(p, -1, None) == mcpu.MCPU_EINVAL and L.kv_pages_share(p, 0, None) == 0
    assert L.kv_page_holders(p, 6) == mcpu.MCPU_EINVAL and L.kv_page_holders(None, 0) == mcpu.MCPU_EINVAL
    # a page is free once its last holder let go; the same id twice in one call stays refused
    assert L.kv_pages_free(p, 2, _i32(1, 1).ctypes.data) == mcpu.MCPU_EINVAL
    assert L.kv_pages_free(p, 4, ids.ctypes.data) == 0
    assert holders() == [1, 2, 0, 0, 0, 0] and L.kv_pool_free_pages(p) == 4
    assert L.kv_pages_free(p, 2, _i32(0, 1).ctypes.data) == 0
    assert L.kv_pages_free(p, 2, _i32(0, 1).ctypes.data) == mcpu.MCPU_EINVAL  # 0 is free: nothing changes
    assert holders() == [0, 1, 0, 0, 0, 0]
    # a page that comes back has one holder again
    assert L.kv_pages_alloc(p, 1, ids.ctypes.data) == 0 and ids[0] == 0 and holders()[0] == 1
    L.kv_pool_destroy(p)


def test_binding_checks_lengths_and_names():
    assert len(mcpu.KERNELS) == 20 and mcpu.KERNELS[14:] == (
        "tree_plan", "tree_attn", "tree_combine", "tree_accept", "tree_commit", "pages_copy")
    with pytest.raises(mcpu.McpuError):
        mcpu.kv_pages_copy([], np.zeros(2, np.int32), np.zeros(2, np.int32), [1], [2], None)


def test_reference_of_a_small_tree():
    """The 64-bit reference itself: visible keys of a small tree by hand, and a path."""
    see = R.visible([-1, 0, 0, 1], 2, 0)
    np.testing.assert_array_equal(see, np.array([[1, 1, 1, 0, 0, 0], [1, 1, 1, 1, 0, 0], [1, 1, 1, 0, 1, 0],
                                                 [1, 1, 1, 1, 0, 1]], bool))
    see = R.visible([-1, 0, 0, 1], 2, 2)
    np.testing.assert_array_equal(see, np.array([[0, 1, 1, 0, 0, 0], [0, 0, 1, 1, 0, 0], [0, 0, 1, 0, 1, 0],
                                                 [0, 0, 0, 1, 0, 1]], bool))
    path, n, following = R.accept(_i32(0, 4), _i32(-1, 0, 0, 2), _i32(9, 5, 6, 7), _i32(6, 1, 7, 3))
    assert path.tolist() == [0, 2, 3, -1] and n.tolist() == [3] and following.tolist() == [3]


# ------------------------------------------------------------------------------ drafting and the engine


def test_lookup_drafts_from_earlier_places():
    from paper_2608_22167_amd.generate import Lookup
    look = Lookup(ngram=2, width=2)
    h = [1, 2, 3, 4, 1, 2, 3, 5, 9, 1, 2]
    # behind (1, 2): 3 5 .. (latest) and 3 4 ..: the 3 is shared
    assert look.tree(h, 10, 2) == ([3, 5, 4], [-1, 0, 0])
    assert look.tree(h, 2, 2) == ([3, 5], [-1, 0])
    assert look.tree(h, 10, 0) == ([], []) and look.tree(h, 0, 5) == ([], [])
    assert look.tree(h + [7], 10, 3) == ([], [])          # 7 never stood anywhere before
    assert look.tree(h + [7, 3], 4, 2) == ([5, 4, 9, 1], [-1, -1, 0, 1])
    assert Lookup().tree([], 5, 5) == ([], []) and Lookup().tree([4], 5, 5) == ([], [])
    # a run that reaches the history's end is shorter
    assert Lookup(1, 1).tree([6, 6], 5, 5) == ([6], [-1])


def test_engine_with_drafts_returns_turns_of_the_asked_length():
    """A stand-in generator whose tokens repeat with period five and whose tree steps confirm what is right."""
    from paper_2608_22167_amd import rollout

    class Seq:
        def __init__(self, sid):
            self.sid, self.history, self.pending = sid, [], []

    class StandIn:
        def __init__(self):
            self.seqs, self.held, self.tree_steps = {}, {}, 0

        def add(self, sid, tokens):
            self.seqs.setdefault(sid, Seq(sid)).pending.extend(tokens)

        def hold(self, sid):
            self.held[sid] = self.seqs[sid].pending[:]
            self.seqs[sid].pending.clear()

        def resume(self, sid, obs):
            self.add(sid, self.held.pop(sid) + list(obs))

        def release(self, sid):
            self.seqs.pop(sid)
            self.held.pop(sid, None)

        @staticmethod
        def token(sid, pos):
            return 100 * sid + pos % 5

        def _draw(self, s):
            t = self.token(s.sid, len(s.history))
            s.pending = [t]
            return t, -1.0

        def step(self):
            out = {}
            for s in self.seqs.values():
                if s.pending:
                    s.history += s.pending
                    out[s.sid] = self._draw(s)
            return out

        def step_tree(self, drafts):
            self.tree_steps += 1
            out = {}
            for s in self.seqs.values():
                if len(s.pending) != 1:
                    continue
                tokens, parents = drafts[s.sid]
                assert len(tokens) <= 7
                s.history += s.pending
                drawn, at = [self._draw(s)], -1
                while True:
                    kids = [i for i, p in enumerate(parents) if p == at and tokens[i] == drawn[-1][0]]
                    if not kids:
                        break
                    at = kids[0]
                    s.history += s.pending
                    drawn.append(self._draw(s))
                out[s.sid] = drawn
            return out

    gen = StandIn()
    eng = rollout.Engine(gen, draft_nodes=7)
    try:
        for turn, n in enumerate((30, 1, 12)):
            futures = {sid: eng.generate(sid, [100 * sid + 9] * 3, n) for sid in (1, 2)}
            for sid, f in futures.items():
                got = f.result(timeout=30)
                assert len(got) == n
        assert gen.tree_steps > 0 and eng.tokens == 2 * (30 + 1 + 12) and eng.steps < eng.tokens / 2
        for sid in (1, 2):
            h = gen.seqs[sid].history
            assert all(h[i] in (100 * sid + 9, gen.token(sid, i)) for i in range(len(h)))
            eng.release(sid).result(timeout=30)
        assert not eng.lookups
    finally:
        eng.close()


def test_tensors_off_the_gpu_are_refused():
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    with pytest.raises(mcpu.McpuError):
        mcpu.tree_accept(i(0, 1), i(-1), i(3), i(4), i(0), i(0), i(0), torch.zeros(256, dtype=torch.uint8))


def test_lookup_fed_in_pieces_drafts_the_same():
    from paper_2608_22167_amd.generate import Lookup
    rng = np.random.default_rng(5)
    tokens = rng.integers(0, 4, 200).tolist()
    pieces, whole = Lookup(), Lookup()
    at = 0
    while at < len(tokens):
        n = int(rng.integers(1, 9))
        pieces.feed(tokens[at:at + n])
        at = min(at + n, len(tokens))
        assert pieces.draft(12, 5) == whole.tree(tokens[:at], 12, 5) == Lookup().tree(tokens[:at], 12, 5)


def test_engine_refuses_drafts_that_no_tree_holds():
    from paper_2608_22167_amd import rollout
    for bad in (-1, mcpu.TREE_MAX_NODES):
        with pytest.raises(ValueError):
            rollout.Engine(None, draft_nodes=bad)


def test_every_tensor_lies_on_the_calls_device(monkeypatch):
    """Stand-ins on GPUs 0 and 1, the current one being 0: no call is made with one argument on the other GPU."""
    made = []

    class Calls:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or mcpu.MCPU_OK

    class Tensor:
        def __init__(self, *shape, dtype=torch.int32, dev=0):
            self.shape, self.dtype, self.dev = torch.Size(shape), dtype, dev
            self.device, self.is_cuda, self.nbytes = torch.device("cuda", dev), True, 4 * self.shape.numel()

        def numel(self):
            return self.shape.numel()

        def get_device(self):
            return self.dev

        is_contiguous = lambda self: True  # noqa: E731
        stride = lambda self: ()           # noqa: E731
        data_ptr = lambda self: D          # noqa: E731

    class Stream:
        def __init__(self, dev):
            self.device_index, self.cuda_stream = dev, 0

    monkeypatch.setattr(mcpu, "lib", Calls)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    s, n = W.TINY, 4
    f32 = dict(dtype=torch.float32)

    def pool(dev=0):
        p = object.__new__(mcpu.KVPool)
        p.shape, p.cfg, p.handle, p.device = s, mcpu.make_cfg(s), None, dev
        p.k = p.v = Tensor(4, **f32, dev=dev)
        return p

    class Weights:
        struct = mcpu.LayerWeights()

        def __init__(self, dev=0):
            self.device = dev

    q = lambda: Tensor(n, s.n_q_heads * s.head_dim, **f32)  # noqa: E731
    x = lambda: Tensor(n, s.hidden, **f32)                  # noqa: E731
    ws, hs, hc = (lambda: Tensor(4096)), _i32(5, 17), _i32(0, 3, 4)
    batch = lambda: [Tensor(2, 8), Tensor(2), Tensor(3)]  # noqa: E731
    calls = {
        "tree_attention": lambda: [s, Tensor(s.n_q_heads, **f32), pool(), *batch(), Tensor(n), hs, hc, q(), q(), ws(), Stream(0)],
        "tree_accept": lambda: [Tensor(3), *[Tensor(n) for _ in range(4)], Tensor(2), Tensor(2), ws(), Stream(0)],
        "kv_tree_commit": lambda: [[pool()], *batch(), Tensor(n), Tensor(2), ws(), Stream(0)],
        "kv_pages_copy": lambda: [[pool()], Tensor(2), Tensor(2), hs, hs, ws(), Stream(0)],
        "decode_layer_tree": lambda: [s, Weights(), pool(), *batch(), Tensor(n), hs, hc, x(), x(), Tensor(n, s.top_k),
                                      Tensor(n, s.top_k, **f32), None, ws(), Stream(0)],
    }
    for name, args in calls.items():
        getattr(mcpu, name)(*args())
        assert made == [name]
        for i, a in enumerate(args()):
            if not isinstance(a, (Tensor, mcpu.KVPool, Weights, Stream, list)):
                continue
            bad = args()
            if isinstance(a, list):
                bad[i] = [pool(), pool(1)]
            elif isinstance(a, (Stream, Weights)):
                bad[i] = type(a)(1)
            elif isinstance(a, mcpu.KVPool):
                bad[i] = pool(1)
            else:
                bad[i].dev = 1
            with pytest.raises(mcpu.McpuError):
                getattr(mcpu, name)(*bad)
        assert made == [name], i
        made.clear()


def test_missing_host_copies_are_refused():
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    for hs, hc in ((None, _i32(0, 1)), (_i32(3), None)):
        with pytest.raises(mcpu.McpuError):
            mcpu.tree_attention(W.TINY, None, None, i(0).view(1, 1), i(3), i(0, 1), i(-1), hs, hc, None, None, None)
