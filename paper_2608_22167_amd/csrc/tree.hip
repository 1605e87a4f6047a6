// Trees of drafted tokens over the paged cache: attention and acceptance.
//
// The n <= 64 nodes of a tree sit in the cache slots behind their sequence's
// committed tokens. Node i stands at position len + depth(i) and attends to the
// committed keys and to its own branch, each inside its window. All nodes of a
// tree read the same committed keys, so the matrix-core columns are (node, query
// head) pairs of one KV head and a page is read once for all of them, where a
// token-by-token step reads it once per token.
//   plan     splits each tree's page range, and finds every node's ancestors
//   attend   one split of one tree and KV head: running maximum, sum and values
//   combine  merges the splits of trees that have several, with the sink
#include "device.h"
#include "kernels_tree.h"

namespace mcpu {

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------

__device__ __forceinline__ int first_page(int len, int window) {
  return (window > 0 ? max(0, len - window + 1) : 0) / PAGE;
}

// Ancestor masks and depths of one tree by one wavefront, lane i = node i, by
// pointer doubling: after round r lane i has the union of its first 2^r ancestors
// and points 2^r steps up. A parent outside [-1, i) raises bit 64 and counts as -1.
__device__ void tree_nodes(const TreePlan& P, int b) {
  const int lane = lane_id();
  const int t0 = P.cu_q[b], n = P.cu_q[b + 1] - t0;
  if (n <= 0 || n > TREE_MAX_NODES || t0 < 0 || t0 + n > P.n_tokens) return;  // raised by the split part
  int up = lane < n ? P.parents[t0 + lane] : -1;
  if (up < -1 || up >= lane) {
    if (lane < n) set_error(P.err, 64);
    up = -1;
  }
  const int parent = up;
  uint64_t seen = 1ull << lane;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    const int from = max(up, 0);
    const uint32_t lo = __shfl((uint32_t)seen, from, 64), hi = __shfl((uint32_t)(seen >> 32), from, 64);
    const int next = __shfl(up, from, 64);
    if (up >= 0) {
      seen |= (uint64_t)hi << 32 | lo;
      up = next;
    }
  }
  const int depth = __popcll(seen) - 1;
  // a window shorter than the branch drops the ancestors that lie window or more steps up
  if (P.window > 0 && __ballot(depth >= P.window) != 0) {
    uint64_t near = 1ull << lane;
    int a = parent;
    for (int k = 1; k < TREE_MAX_NODES; ++k) {
      if (a >= 0 && k < P.window) near |= 1ull << a;
      const int next = __shfl(parent, max(a, 0), 64);
      a = a >= 0 ? next : -1;
    }
    seen = near;
  }
  if (lane < n) {
    TreeNode d;
    d.seen = seen;
    d.depth = depth;
    d.pad = 0;
    P.node[t0 + lane] = d;
    P.tok_seq[t0 + lane] = b;
  }
}

// Exclusive prefix of `local` over the block's threads, and the total.
__device__ int plan_scan(int local, int* sums, int& total) {
  const int incl = wave_incl_scan(local), wave = threadIdx.x >> 6, lane = lane_id(), nw = blockDim.x >> 6;
  __syncthreads();  // sums may still be read for the scan before
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < nw; ++w) {
    before += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  return before + incl - local;
}

// Workgroup 0: the splits, a thread per sequence. Workgroups 1..: the nodes, a
// wavefront per sequence. Bound by latency.
__global__ __launch_bounds__(1024) void tree_plan_kernel(TreePlan P) {
  if (blockIdx.x > 0) {
    const int b = (blockIdx.x - 1) * 16 + uniform(threadIdx.x >> 6);
    if (b < P.batch) tree_nodes(P, b);
    return;
  }
  __shared__ int sums[16];
  int items = 0, rows = 0;
  for (int base = 0; base < P.batch; base += blockDim.x) {
    const int b = base + threadIdx.x;
    TreeItem it{};
    int np = 0;
    if (b < P.batch) {
      it.b = b;
      it.t0 = P.cu_q[b];
      it.n = P.cu_q[b + 1] - it.t0;
      it.len = P.seq_lens[b];
      if (it.n < 0 || it.n > TREE_MAX_NODES || it.t0 < 0 || it.t0 + it.n > P.n_tokens || it.len < 0 ||
          (it.n > 0 && (it.len + it.n - 1) / PAGE >= P.max_pages)) {
        set_error(P.err, 8);
        it.n = 0;
      }
      if (it.n > 0) {
        np = (it.len + it.n - 1) / PAGE - first_page(it.len, P.window) + 1;
        it.splits = (np + P.pps - 1) / P.pps;
      }
    }
    int all_items, all_rows;
    const int at = items + plan_scan(it.splits, sums, all_items);
    it.row0 = rows + plan_scan(it.splits > 1 ? it.splits * it.n : 0, sums, all_rows);
    items += all_items;
    rows += all_rows;
    if (b < P.batch) {
      P.seq_split[b] = make_int2(it.row0, it.splits);
      const int first = first_page(it.len, P.window), n_splits = it.splits;
      const int row0 = it.row0;
      for (int k = 0; k < n_splits && at + k < P.n_items; ++k) {  // the pages shared out evenly
        it.pg0 = first + (int)((int64_t)k * np / n_splits);
        it.pg1 = first + (int)((int64_t)(k + 1) * np / n_splits);
        it.row0 = row0 + k * it.n;
        P.item[at + k] = it;
      }
    }
  }
  if (threadIdx.x == 0 && (items != P.n_items || rows != P.n_rows)) set_error(P.err, 8);
}

hipError_t launch_tree_plan(const TreePlan& p, hipStream_t s) {
  hipLaunchKernelGGL(tree_plan_kernel, dim3(1 + (p.batch + 15) / 16), dim3(1024), 0, s, p);
  return hipGetLastError();
}

// An item's record, every field checked before it addresses memory: where the
// device arrays disagree with the host's plan it may be stale.
__device__ __forceinline__ bool load_item(const TreeAttn& P, int i, TreeItem& it) {
  it = P.item[i];
  it.b = uniform(it.b); it.t0 = uniform(it.t0); it.n = uniform(it.n); it.len = uniform(it.len);
  it.pg0 = uniform(it.pg0); it.pg1 = uniform(it.pg1); it.row0 = uniform(it.row0); it.splits = uniform(it.splits);
  const bool ok = it.b >= 0 && it.b < P.batch && it.n > 0 && it.n <= TREE_MAX_NODES && it.t0 >= 0 &&
                  it.t0 + it.n <= P.n_tokens && it.len >= 0 && it.pg0 >= 0 && it.pg0 < it.pg1 &&
                  it.pg1 <= P.max_pages && (it.splits == 1 || (it.row0 >= 0 && it.row0 + it.n <= P.n_rows));
  if (!ok && lane_id() == 0) set_error(P.err, 8);
  return ok;
}

// ---------------------------------------------------------------------------
// attend, any type and head dim: 16 columns per wavefront
// ---------------------------------------------------------------------------

// zero the values that are not finite; true if there were any
__device__ __forceinline__ bool drop_nonfinite(uint32_t& w) {
  const bool lo = (w & 0x7F80u) == 0x7F80u, hi = (w & 0x7F800000u) == 0x7F800000u;
  w &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0x0000FFFFu : 0xFFFFFFFFu);
  return lo || hi;
}
__device__ __forceinline__ bool drop_nonfinite(float& f) {
  const bool bad = (__float_as_uint(f) & 0x7F800000u) == 0x7F800000u;
  f = bad ? 0.f : f;
  return bad;
}
__device__ __forceinline__ bool drop_nonfinite(Frag4<bf16>& f) {
  const bool a = drop_nonfinite(f.v.x), b = drop_nonfinite(f.v.y);
  return a || b;
}
__device__ __forceinline__ bool drop_nonfinite(Frag4<float>& f) {
  const bool a = drop_nonfinite(f.v.x), b = drop_nonfinite(f.v.y), c = drop_nonfinite(f.v.z), d = drop_nonfinite(f.v.w);
  return a || b || c || d;
}

// What a column (a node and one of its heads) sees: committed keys from lo, and
// the nodes in `seen`.
struct Sight {
  int lo;
  uint64_t seen;
  __device__ __forceinline__ bool key(int slot, int len, int n) const {
    const int a = slot - len;
    const bool old = slot >= lo, mine = (a < n) & ((seen >> (a & 63) & 1) != 0);
    return a < 0 ? old : mine;
  }
};
__device__ __forceinline__ Sight sight_of(const TreeAttn& P, const TreeItem& it, int node) {
  const TreeNode d = P.node[it.t0 + node];
  Sight s;
  s.lo = P.window > 0 ? it.len + d.depth - P.window + 1 : 0;
  s.seen = d.seen;
  return s;
}

// One wavefront per (split, KV head, 16 columns). As everywhere in this library
// a page's scores S^T = K q^T are one 16x16 tile with keys as rows, in the lane
// layout that the value product O^T += V^T P^T takes; the softmax runs online in
// base 2. Pages past the committed keys, left of a node's window or missing are
// masked; on such pages values that are not finite are taken out of the value
// product (a weight of zero times infinity is not zero) and added to the columns
// that see them.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_attn_kernel(TreeAttn P, int tiles) {
  const int lane = lane_id(), hl = lane & 15, grp = lane >> 4;
  const unsigned id = blockIdx.x * 4 + uniform(threadIdx.x >> 6), hkv = P.hkv;
  const int g = id % hkv, tile = id / hkv % (unsigned)tiles, i = id / hkv / (unsigned)tiles;
  if (i >= P.n_items) return;  // no barriers below
  TreeItem it;
  if (!load_item(P, i, it)) return;
  const int G = P.hq / P.hkv, cols = it.n * G;
  if (16 * tile >= cols) return;
  const int c = 16 * tile + hl, node = min(c / G, it.n - 1), head = g * G + c % G;
  const bool valid = c < cols;
  const Sight sight = sight_of(P, it, node);
  Frag<T> qf[D / 32];
  const T* qb = reinterpret_cast<const T*>(P.q) + ((int64_t)(it.t0 + node) * P.hq + head) * D + 8 * grp;
#pragma unroll
  for (int cc = 0; cc < D / 32; ++cc) {
    qf[cc].load(qb + 32 * cc);
    qf[cc].keep_if(valid);
  }
  const T* kpool = reinterpret_cast<const T*>(P.k_pool);
  const T* vpool = reinterpret_cast<const T*>(P.v_pool);
  const int32_t* ptab = P.page_table + (int64_t)it.b * P.max_pages;
  const int64_t head_off = (int64_t)g * PAGE * D, page_elems = (int64_t)P.hkv * PAGE * D;

  struct Page {
    Frag<T> k[D / 32];
    Frag4<T> v[D / 16];
    const T* vp;
    bool ok;
  };
  auto fetch = [&](Page& p, int pg) {
    int pid = uniform(ptab[min(pg, it.pg1 - 1)]);
    p.ok = pid >= 0 && pid < P.n_pages;
    if (!p.ok && pg < it.pg1 && lane == 0) set_error(P.err, 1);
    pid = p.ok ? pid : 0;
    const T* kp = kpool + pid * page_elems + head_off;
    p.vp = vpool + pid * page_elems + head_off;
#pragma unroll
    for (int cc = 0; cc < D / 32; ++cc) p.k[cc].load(kp + (64 * cc + lane) * 8);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) p.v[n].load(p.vp + (64 * n + lane) * 4);
  };
  float m = -INFINITY, l = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};

  Page cur, nxt;
  fetch(cur, it.pg0);
  for (int pg = it.pg0; pg < it.pg1; ++pg) {
    fetch(nxt, pg + 1);
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int cc = 0; cc < D / 32; ++cc) sc = mma32(cur.k[cc], qf[cc], sc);
    const int k0 = pg * PAGE;
    const bool edge = k0 + PAGE > it.len || (P.window > 0 && k0 < it.len + it.n - P.window) || !cur.ok;
    float x[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = sc[r] * P.scale_log2;
    bool odd = false;
    if (edge) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool in = sight.key(k0 + 4 * grp + r, it.len, it.n) & cur.ok;
        x[r] = in ? x[r] : -INFINITY;
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) odd = drop_nonfinite(cur.v[n]) || odd;
    }
    float mloc = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    mloc = fmaxf(mloc, __shfl_xor(mloc, 16, 64));
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32, 64));
    const float m_new = fmaxf(m, mloc);
    const float m_sub = m_new == -INFINITY ? 0.f : m_new;  // no key seen yet: all weights 2^-inf
    const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
    float pr[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) pr[r] = __builtin_amdgcn_exp2f(x[r] - m_sub);
    l *= alpha;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      acc[n] *= alpha;
      acc[n] = mma16_p(cur.v[n], pr, acc[n], n == 0 ? &l : nullptr);
    }
    m = m_new;
    if (edge && cur.ok && __ballot(odd) != 0) {  // rare: values that are not finite, for the columns that see them
      for (int s = 0; s < PAGE; ++s) {
        if (!sight.key(k0 + s, it.len, it.n)) continue;
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float v = Elem<T>::load(cur.vp, v_off(s, 16 * n + 4 * grp + r));
            float w = v;
            if (drop_nonfinite(w)) acc[n][r] += v;
          }
      }
    }
    cur = nxt;
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (!valid) return;
  if (it.splits > 1) {
    const int64_t row = (int64_t)(it.row0 + node) * P.hq + head;
    if (grp == 0) *reinterpret_cast<float2*>(P.part_ml + 2 * row) = make_float2(m, l);
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
      *reinterpret_cast<float4*>(P.part_acc + row * D + 16 * n + 4 * grp) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
    return;
  }
  // o = 2^(m - M) acc / (2^(sink log2e - M) + 2^(m - M) l), M = max(sink log2e, m); no key and no sink: zeros
  float f = 1.0f;
  if (P.sinks) {
    const float sk = P.sinks[head] * LOG2E, M = fmaxf(m, sk);
    f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
    l = l * f + __builtin_amdgcn_exp2f(sk - M);
  }
  T* o = reinterpret_cast<T*>(P.o) + ((int64_t)(it.t0 + node) * P.hq + head) * D + 4 * grp;
#pragma unroll
  for (int n = 0; n < D / 16; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) Elem<T>::store(o, 16 * n + r, l == 0.f ? 0.f : f * acc[n][r] / l);
}

template <typename T, int D>
static hipError_t tree_attn_impl(const TreeAttn& p, hipStream_t s) {
  const int tiles = (p.max_nodes * (p.hq / p.hkv) + 15) / 16;
  const int64_t waves = (int64_t)p.n_items * p.hkv * tiles;
  if (waves > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL((tree_attn_kernel<T, D>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p, tiles);
  return hipGetLastError();
}

hipError_t launch_tree_attn(int dtype, int head_dim, const TreeAttn& p, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  if (dtype == 0) return head_dim == 32 ? tree_attn_impl<float, 32>(p, s) : tree_attn_impl<float, 64>(p, s);
  return head_dim == 32 ? tree_attn_impl<bf16, 32>(p, s) : tree_attn_impl<bf16, 64>(p, s);
}

// ---------------------------------------------------------------------------
// combine: o_h = sum_s 2^(m_s - M) acc_s / (2^(sink_h log2e - M) + sum_s 2^(m_s - M) l_s)
// ---------------------------------------------------------------------------

// A wavefront per (node, head) of the trees with several splits, D / 4 lanes per
// partial row: 256 / D rows per load, lane groups joined at the end.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeCombine P) {
  constexpr int LR = D / 4, RW = 64 / LR;
  const int lane = lane_id(), sub = lane / LR, dim = 4 * (lane % LR);
  const unsigned id = blockIdx.x * 4 + uniform(threadIdx.x >> 6), hq = P.hq;
  const int t = id / hq, h = id % hq;
  if (t >= P.n_tokens) return;
  const int b = uniform(P.tok_seq[t]);
  if (b < 0 || b >= P.batch) return;  // arrays that disagree with the plan (error bit set there)
  const int2 sp = P.seq_split[b];
  const int row0 = uniform(sp.x), splits = uniform(sp.y);
  const int t0 = uniform(P.cu_q[b]), n = uniform(P.cu_q[b + 1]) - t0, node = t - t0;
  if (splits <= 1 || node < 0 || node >= n || row0 < 0 || (int64_t)row0 + (int64_t)splits * n > P.n_rows) return;
  float M = -INFINITY, L = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = sub; k < splits; k += RW) {
    const int64_t row = (int64_t)(row0 + k * n + node) * P.hq + h;
    const float2 ml = *reinterpret_cast<const float2*>(P.part_ml + 2 * row);
    const float4 v = *reinterpret_cast<const float4*>(P.part_acc + row * D + dim);
    const float Mn = fmaxf(M, ml.x), sub_m = Mn == -INFINITY ? 0.f : Mn;
    const float r = __builtin_amdgcn_exp2f(M - sub_m), f = __builtin_amdgcn_exp2f(ml.x - sub_m);
    L = L * r + ml.y * f;
    a.x = a.x * r + v.x * f; a.y = a.y * r + v.y * f; a.z = a.z * r + v.z * f; a.w = a.w * r + v.w * f;
    M = Mn;
  }
  // join the lane groups, then the sink
  float Mt = M;
#pragma unroll
  for (int o = LR; o < 64; o <<= 1) Mt = fmaxf(Mt, __shfl_xor(Mt, o, 64));
  if (P.sinks) Mt = fmaxf(Mt, P.sinks[h] * LOG2E);
  const float f = __builtin_amdgcn_exp2f(M - (Mt == -INFINITY ? 0.f : Mt));
  L *= f;
  a.x *= f; a.y *= f; a.z *= f; a.w *= f;
#pragma unroll
  for (int o = LR; o < 64; o <<= 1) {
    L += __shfl_xor(L, o, 64);
    a.x += __shfl_xor(a.x, o, 64);
    a.y += __shfl_xor(a.y, o, 64);
    a.z += __shfl_xor(a.z, o, 64);
    a.w += __shfl_xor(a.w, o, 64);
  }
  if (P.sinks) L += __builtin_amdgcn_exp2f(P.sinks[h] * LOG2E - Mt);
  if (sub != 0) return;
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  store4(reinterpret_cast<T*>(P.o) + ((int64_t)t * P.hq + h) * D + dim,
         make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
}

hipError_t launch_tree_combine(int dtype, int head_dim, const TreeCombine& p, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  if ((int64_t)p.n_tokens * p.hq > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(((int64_t)p.n_tokens * p.hq + 3) / 4)), block(256);
  if (dtype == 0) {
    if (head_dim == 32) hipLaunchKernelGGL((tree_combine_kernel<float, 32>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_combine_kernel<float, 64>), grid, block, 0, s, p);
  } else {
    if (head_dim == 32) hipLaunchKernelGGL((tree_combine_kernel<bf16, 32>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_combine_kernel<bf16, 64>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// accept
// ---------------------------------------------------------------------------

// One wavefront per tree, lane i = node i. From the root (node 0) the walk goes to
// the lowest child whose drafted id equals the draw at its parent: one ballot per
// step, at most 64 steps (a child comes after its parent). Bound by latency.
__global__ __launch_bounds__(64) void tree_accept_kernel(TreeAccept P) {
  const int b = blockIdx.x, lane = lane_id();
  const int t0 = P.cu_q[b], n = P.cu_q[b + 1] - t0;
  int count = 0, last = -1;
  if (n < 0 || n > TREE_MAX_NODES || t0 < 0 || t0 + n > P.n_tokens) {
    if (lane == 0) set_error(P.err, 8);
  } else if (n > 0) {
    const bool in = lane < n;
    const int parent = in ? P.parents[t0 + lane] : -1;
    const int draft = in ? P.draft[t0 + lane] : 0, sampled = in ? P.sampled[t0 + lane] : 0;
    if (in && (parent < -1 || parent >= lane)) set_error(P.err, 64);
    int cur = 0, mine = -1;
    while (true) {
      if (lane == count) mine = cur;
      ++count;
      last = __builtin_amdgcn_readlane(sampled, cur);
      const uint64_t hit = __ballot(in && lane > cur && parent == cur && draft == last);
      if (hit == 0) break;
      cur = (int)__builtin_ctzll(hit);
    }
    if (in) P.path[t0 + lane] = mine;
  }
  if (lane == 0) {
    P.n_path[b] = count;
    P.next[b] = last;
  }
}

hipError_t launch_tree_accept(const TreeAccept& p, hipStream_t s) {
  if (p.batch == 0) return hipSuccess;
  hipLaunchKernelGGL(tree_accept_kernel, dim3(p.batch), dim3(64), 0, s, p);
  return hipGetLastError();
}

}  // namespace mcpu
