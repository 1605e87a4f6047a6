"""Drafted token trees in 64 bits, written from the definitions in mcpu.h with
dense arrays and loops: visible keys, attention with its error bound, the
accepted path and its commit."""
import numpy as np

PAGE = 16


def depths(parents):
    d = []
    for i, p in enumerate(parents):
        d.append(0 if p < 0 else d[p] + 1)
    return np.array(d, np.int64)


def visible(parents, length, window):
    """[n, length + n] truth table: key slot j of node i."""
    n, d = len(parents), depths(parents)
    see = np.zeros((n, length + n), bool)
    for i in range(n):
        pos = length + d[i]
        lo = max(0, pos - window + 1) if window else 0
        see[i, lo:length] = True
        a = i
        while a >= 0:
            see[i, length + a] = not window or length + d[a] > pos - window
            a = parents[a]
    return see


def slot_offsets(d):
    """Element offsets of (slot, dim) in one KV head's block of a K and of a V page."""
    s, i = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    return ((i // 8) * PAGE + s) * 8 + i % 8, (((i // 16) * 4 + s // 4) * 16 + i % 16) * 4 + s % 4


def keys_of(pool, offsets, table, upto):
    """Keys (or values) of slots 0 .. upto - 1 of one sequence as [Hkv, upto, d]
    float64 from a pool [pages, Hkv, 16 * d]; slots of missing pages are zero, and
    `there` says which are not."""
    n_pages, hkv, _ = pool.shape
    out = np.zeros((hkv, upto, offsets.shape[1]))
    there = np.zeros(upto, bool)
    for j in range(upto):
        p = table[j // PAGE]
        if 0 <= p < n_pages:
            out[:, j] = pool[p][:, offsets[j % PAGE]]
            there[j] = True
    return out, there


def attention(q, k_pool, v_pool, table, seq_lens, cu_q, parents, sinks, window, bf16):
    """q [T, Hq, d] and pools [pages, Hkv, 16 * d] float64. Returns o [T, Hq, d]
    and how far a kernel may be from it:

    a weight w_j is off by a factor of at most 1 + e_w, where the score's error is
    that of d + 4 roundings to 24 bits of sum |q_i k_i| / sqrt(d), the base-2
    exponential's a few 2^-23, and a bf16 layer rounds the weight itself (2^-8).
    Weights stand in numerator and normaliser, so o moves by up to 2 e_w sum w |v|,
    by n roundings of the sums over n keys, and by its own rounding."""
    T, hq, d = q.shape
    hkv = k_pool.shape[1]
    G = hq // hkv
    ko, vo = slot_offsets(d)
    out, tol = np.zeros_like(q), np.zeros_like(q)
    for b in range(len(seq_lens)):
        t0, n, L = int(cu_q[b]), int(cu_q[b + 1] - cu_q[b]), int(seq_lens[b])
        if n == 0:
            continue
        K, there = keys_of(k_pool, ko, table[b], L + n)
        V, _ = keys_of(v_pool, vo, table[b], L + n)
        see = visible(parents[t0:t0 + n], L, window) & there
        for h in range(hq):
            qh = q[t0:t0 + n, h]
            with np.errstate(invalid="ignore", over="ignore"):
                z = qh @ K[h // G].T / np.sqrt(d)
                size = np.abs(qh) @ np.abs(K[h // G]).T / np.sqrt(d)
            s = -np.inf if sinks is None else float(sinks[h])
            for i in range(n):
                zi = z[i, see[i]]
                m = max(s, zi.max(initial=-np.inf))
                if m == -np.inf:
                    continue  # no key and no sink: zeros
                w = np.exp(zi - m)
                w = w / (w.sum() + np.exp(s - m))
                v = V[h // G][see[i]]
                out[t0 + i, h] = w @ v
                e_w = (d + 4) * 2.0 ** -24 * size[i, see[i]].max(initial=0) + 2.0 ** -20 + (2.0 ** -8 if bf16 else 0)
                tol[t0 + i, h] = (2 * e_w * (1 + e_w) + 2 * (len(zi) + 8) * 2.0 ** -24) * (w @ np.abs(v))
    eps = 2.0 ** -8 if bf16 else 2.0 ** -24
    return out, tol + eps * (np.abs(out) + tol) + 1e-30


def accept(cu_q, parents, draft, sampled):
    path = np.full(len(parents), -1, np.int32)
    n_path = np.zeros(len(cu_q) - 1, np.int32)
    following = np.full(len(cu_q) - 1, -1, np.int32)
    for b in range(len(cu_q) - 1):
        t0, n = int(cu_q[b]), int(cu_q[b + 1] - cu_q[b])
        cur = 0 if n else None
        while cur is not None:
            path[t0 + n_path[b]] = cur
            n_path[b] += 1
            following[b] = sampled[t0 + cur]
            cur = next((c for c in range(cur + 1, n) if parents[t0 + c] == cur and draft[t0 + c] == following[b]), None)
    return path, n_path, following


def commit(pool, offsets, table, seq_lens, cu_q, path, n_path):
    """A pool [pages, Hkv, 16 * d] after the accepted paths moved."""
    new = pool.copy()
    for b in range(len(seq_lens)):
        for i in range(int(n_path[b])):
            s, t = int(seq_lens[b] + path[cu_q[b] + i]), int(seq_lens[b]) + i
            ps, pt = table[b, s // PAGE], table[b, t // PAGE]
            if ps >= 0 and pt >= 0:
                new[pt][:, offsets[t % PAGE]] = pool[ps][:, offsets[s % PAGE]]
    return new


def random_tree(rng, n, reach=4):
    """Parents of n nodes: node 0 a root, the others behind one of the `reach` nodes before them."""
    return [-1] + [int(rng.integers(max(0, i - reach), i)) for i in range(1, n)] if n else []
