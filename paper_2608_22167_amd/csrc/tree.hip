// Trees of drafted tokens over the paged cache: attention and acceptance.
//
// The n <= 64 nodes of a tree sit in the cache slots behind their sequence's
// committed tokens. Node i stands at position len + depth(i) and attends to the
// committed keys and to its own branch, each inside its window. All nodes of a
// tree read the same committed keys, so the matrix-core columns are (node, query
// head) pairs of one KV head and a page is read once for all of them, where a
// token-by-token step reads it once per token.
//   plan     splits each tree's page range (large split batches only: else each
//            wavefront finds its split)
//   attend   one split of one tree and KV head: the nodes' ancestors, running maximum,
//            sum and values
//   combine  merges the splits of trees that have several, with the sink
#include <type_traits>

#include "device.h"
#include "kernels_tree.h"

namespace mcpu {

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------------------
// plan: which pages of which tree a workgroup attends to
// ---------------------------------------------------------------------------

__device__ __forceinline__ int first_page(int len, int window) {
  return (window > 0 ? max(0, len - window + 1) : 0) / PAGE;
}

// Sequence b's tree, its pages and its splits; none for an empty tree, for b past
// the batch and for device arrays that do not fit the call (`bad`, reported as bit 8).
struct TreeSpan {
  int t0, n, len, pages, splits;
  bool bad;
};
__device__ __forceinline__ TreeSpan tree_span(const TreeArgs& P, int b) {
  const int at = min(b, P.batch - 1);  // loads without a branch, so that several spans' are in flight together
  TreeSpan s;
  s.t0 = P.cu_q[at];
  s.n = P.cu_q[at + 1] - s.t0;
  s.len = P.seq_lens[at];
  s.bad = s.n < 0 || s.n > P.max_nodes || s.t0 < 0 || s.t0 > P.n_tokens - s.n || s.len < 0 ||
          (s.n > 0 && (s.len > INT32_MAX - TREE_MAX_NODES || (s.len + s.n - 1) / PAGE >= P.max_pages));
  s.n = s.bad || b >= P.batch ? 0 : s.n;
  s.pages = s.n > 0 ? (s.len + s.n - 1) / PAGE - first_page(s.len, P.window) + 1 : 0;
  s.splits = (s.pages + P.pps - 1) / P.pps;
  return s;
}
// partial rows of a tree: its nodes once per split, if there are several
__device__ __forceinline__ int rows_of(const TreeSpan& s) { return s.splits > 1 ? s.splits * s.n : 0; }

// Split k of a tree, whose pages the splits share evenly.
__device__ __forceinline__ TreeItem split_of(const TreeArgs& P, const TreeSpan& s, int b, int row0, int k) {
  const int first = first_page(s.len, P.window);
  TreeItem it;
  it.b = b; it.t0 = s.t0; it.n = s.n; it.len = s.len; it.splits = s.splits;
  it.pg0 = first + (int)((int64_t)k * s.pages / s.splits);
  it.pg1 = first + (int)((int64_t)(k + 1) * s.pages / s.splits);
  it.row0 = row0 + k * s.n;
  return it;
}

// Has a tree whose first split is item `at`, and whose first partial row is row0, a
// place in the host's plan? One that has not (device arrays that disagree with the
// host's) is left out as a whole.
__device__ __forceinline__ bool placed(const TreeArgs& P, const TreeSpan& s, int at, int row0) {
  return s.n > 0 && at >= 0 && at <= P.n_items - s.splits && row0 >= 0 && row0 <= P.n_rows - rows_of(s);
}

// The plan of a large batch, by one workgroup: a thread per sequence, and the
// records of a wavefront's 64 trees written together, lane j the j-th. Where the
// device's arrays disagree with the host's plan, the records that no tree has and all
// rows are marked as such, since an earlier call may have left others there.
__global__ __launch_bounds__(1024) void tree_plan_kernel(TreeArgs P, TreeItem* out) {
  __shared__ int sums[2][16];
  __shared__ int bad;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const bool covered = P.cu_q[0] == 0 && P.cu_q[P.batch] == P.n_tokens;
  if (threadIdx.x == 0) bad = !covered;
  int items = 0, rows = 0;
  for (int base = 0; base < P.batch; base += 1024) {
    const int b = base + threadIdx.x;
    const TreeSpan s = tree_span(P, b);
    const int incl = wave_incl_scan(s.splits), rincl = wave_incl_scan(rows_of(s));
    __syncthreads();  // sums may still be read for the tile before
    if (s.bad) bad = 1;
    if (lane == 63) {
      sums[0][wave] = incl;
      sums[1][wave] = rincl;
    }
    __syncthreads();
    int at = items, row0 = rows + rincl - rows_of(s);
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? sums[0][w] : 0;
      row0 += w < wave ? sums[1][w] : 0;
      items += sums[0][w];
      rows += sums[1][w];
    }
    const int in = placed(P, s, at + incl - s.splits, row0);
    const int all = __shfl(incl, 63, 64);
    for (int j0 = 0; j0 < all; j0 += 64) {
      const int j = j0 + lane;
      int o = 0;  // the first lane with incl > j: the tree of record j
#pragma unroll
      for (int step = 32; step; step >>= 1) o += __shfl(incl, o + step - 1, 64) <= j ? step : 0;
      const int src = min(o, 63);
      TreeSpan r;
      r.t0 = __shfl(s.t0, src, 64); r.n = __shfl(s.n, src, 64); r.len = __shfl(s.len, src, 64);
      r.pages = __shfl(s.pages, src, 64); r.splits = __shfl(s.splits, src, 64);
      const int k = j - (__shfl(incl, src, 64) - r.splits), rb = __shfl(b, src, 64), rr = __shfl(row0, src, 64);
      const int rin = __shfl(in, src, 64);
      if (j < all && at + j >= 0 && at + j < P.n_items) out[at + j] = split_of(P, r, rin ? rb : -1, rr, k);
    }
  }
  __syncthreads();
  if (!bad && items == P.n_items && rows == P.n_rows) return;
  if (threadIdx.x == 0) set_error(P.err, 8);
  for (int i = max(0, items) + threadIdx.x; i < P.n_items; i += 1024) out[i].b = -1;
  for (int t = threadIdx.x; t < P.n_tokens; t += 1024) P.tok[t] = make_int4(0, 0, 0, 0);
}

hipError_t launch_tree_plan(const TreeArgs& p, TreeItem* out, hipStream_t s) {
  hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(1024), 0, s, p, out);
  return hipGetLastError();
}

// Item i of the step, for a whole wavefront; false if there is none (an empty tree,
// or device arrays that disagree with the host's plan: bit 8). Where no tree is
// split, item i is tree i. Otherwise, up to TREE_SCAN sequences, each wavefront
// finds it by itself, four sequences per lane: one round of memory instead of a
// launch in front of the step (48 trees 7 us, one tree 5 us). Larger batches read
// the plan kernel's records, every field checked before it addresses memory.
__device__ __forceinline__ bool find_item(const TreeArgs& P, int i, TreeItem& it) {
  bool ok = false;
  it = TreeItem{};
  if (P.n_rows == 0) {
    const TreeSpan s = tree_span(P, i);
    if (s.bad) set_error(P.err, 8);
    if (uniform(s.n) == 0) return false;
    it = split_of(P, s, i, 0, 0);
    ok = it.splits == 1;
  } else if (P.item) {
    it = P.item[i];
    ok = it.b >= 0 && it.b < P.batch && it.n > 0 && it.n <= TREE_MAX_NODES && it.t0 >= 0 &&
         it.t0 <= P.n_tokens - it.n && it.len >= 0 && it.pg0 >= 0 && it.pg0 < it.pg1 && it.pg1 <= P.max_pages &&
         it.splits > 0 && (it.splits == 1 || (it.row0 >= 0 && it.row0 <= P.n_rows - it.n));
  } else {
    const int lane = lane_id();
    TreeSpan s[TREE_SCAN / 64];
#pragma unroll
    for (int c = 0; c < TREE_SCAN / 64; ++c) s[c] = tree_span(P, 64 * c + lane);
    int items = 0, rows = 0, end = 0;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < TREE_SCAN / 64; ++c) {
      if (64 * c >= P.batch) break;
      const int incl = wave_incl_scan(s[c].splits), rincl = wave_incl_scan(rows_of(s[c]));
      const bool in = placed(P, s[c], items + incl - s[c].splits, rows + rincl - rows_of(s[c]));
      const uint64_t past = __ballot(items + incl > i);
      if (it.n == 0 && past != 0) {  // uniform
        const int src = (int)__builtin_ctzll(past);
        TreeSpan r;
        r.t0 = __builtin_amdgcn_readlane(s[c].t0, src); r.n = __builtin_amdgcn_readlane(s[c].n, src);
        r.len = __builtin_amdgcn_readlane(s[c].len, src); r.pages = __builtin_amdgcn_readlane(s[c].pages, src);
        r.splits = __builtin_amdgcn_readlane(s[c].splits, src);
        const int k = i - (items + __builtin_amdgcn_readlane(incl, src) - r.splits);
        it = split_of(P, r, 64 * c + src, rows + __builtin_amdgcn_readlane(rincl, src) - rows_of(r), k);
        ok = __builtin_amdgcn_readlane(in, src);
      }
      items += __builtin_amdgcn_readlane(incl, 63);
      rows += __builtin_amdgcn_readlane(rincl, 63);
      end = __builtin_amdgcn_readlane(s[c].t0 + s[c].n, min(P.batch - 1 - 64 * c, 63));
      bad |= s[c].bad;
      s[c].n = in ? s[c].n : 0;
    }
    const bool covered = __builtin_amdgcn_readlane(s[0].t0, 0) == 0 && end == P.n_tokens;
    if (i == 0 && (__ballot(bad) != 0 || !covered || items != P.n_items || rows != P.n_rows)) {
      // rare: the rows of no tree are marked as such, as an earlier call may have left records there
      if (lane == 0) set_error(P.err, 8);
      for (int t = lane; t < P.n_tokens + lane; t += 64) {
        bool mine = false;
#pragma unroll
        for (int c = 0; c < TREE_SCAN / 64; ++c)
          for (int src = 0; src < 64; ++src)
            mine |= (uint32_t)(t - __builtin_amdgcn_readlane(s[c].t0, src)) < (uint32_t)__builtin_amdgcn_readlane(s[c].n, src);
        if (!mine && t < P.n_tokens) P.tok[t] = make_int4(0, 0, 0, 0);
      }
    }
  }
  it.b = uniform(it.b); it.t0 = uniform(it.t0); it.n = uniform(it.n); it.len = uniform(it.len);
  it.pg0 = uniform(it.pg0); it.pg1 = uniform(it.pg1); it.row0 = uniform(it.row0); it.splits = uniform(it.splits);
  if (!ok && lane_id() == 0) set_error(P.err, 8);
  return ok;
}

// The ancestors of a tree's nodes by one wavefront, lane i = node i: bit a of
// `seen` is set if node a is an ancestor of i, or i itself, inside i's window;
// depth counts all ancestors. By pointer doubling: after round r lane i has the
// union of its first 2^r ancestors and points 2^r steps up. A parent outside
// [-1, i) raises bit 64 and counts as -1.
struct Nodes {
  uint64_t seen;
  int depth;
};
__device__ __forceinline__ int parent_of(const TreeArgs& P, const TreeItem& it) {
  const int lane = lane_id();
  return lane < it.n ? P.parents[it.t0 + lane] : -1;
}
__device__ __forceinline__ Nodes nodes_of(const TreeArgs& P, const TreeItem& it, int up) {  // up = parent_of(P, it)
  const int lane = lane_id();
  if (up < -1 || up >= lane) {
    if (lane < it.n) set_error(P.err, 64);
    up = -1;
  }
  const int parent = up;
  Nodes d;
  d.seen = 1ull << lane;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    if (__ballot(up >= 0) == 0) break;
    const int from = max(up, 0);
    const uint32_t lo = __shfl((uint32_t)d.seen, from, 64), hi = __shfl((uint32_t)(d.seen >> 32), from, 64);
    const int next = __shfl(up, from, 64);
    d.seen |= up >= 0 ? (uint64_t)hi << 32 | lo : 0;
    up = up >= 0 ? next : -1;
  }
  d.depth = __popcll(d.seen) - 1;
  // a window shorter than the branch drops the ancestors that lie window or more steps up
  if (P.window > 0 && __ballot(d.depth >= P.window) != 0) {
    uint64_t near = 1ull << lane;
    int a = parent;
    for (int k = 1; k < TREE_MAX_NODES; ++k) {
      near |= a >= 0 && k < P.window ? 1ull << (a & 63) : 0;
      const int next = __shfl(parent, max(a, 0), 64);
      a = a >= 0 ? next : -1;
    }
    d.seen = near;
  }
  return d;
}

// The positions at which a layer rotates its nodes, a wavefront per tree. Bound by
// latency (3 us).
__global__ __launch_bounds__(256) void tree_positions_kernel(TreeArgs P, int32_t* rope) {
  const int b = blockIdx.x * 4 + uniform(threadIdx.x >> 6), lane = lane_id();
  if (b >= P.batch) return;
  const TreeSpan s = tree_span(P, b);
  if (s.bad) set_error(P.err, 8);
  TreeItem it{};
  it.t0 = uniform(s.t0);
  it.n = uniform(s.n);
  const Nodes d = nodes_of(P, it, parent_of(P, it));
  if (lane < it.n) rope[it.t0 + lane] = s.len + d.depth;
}

hipError_t launch_tree_positions(const TreeArgs& p, int32_t* rope, hipStream_t s) {
  hipLaunchKernelGGL(tree_positions_kernel, dim3((p.batch + 3) / 4), dim3(256), 0, s, p, rope);
  return hipGetLastError();
}

// What the combine needs to know of a tree's tokens: the first partial row, the
// rows from one split to the next, and the splits. Written by one wavefront of the
// tree's first split, in steps that have a combine.
__device__ __forceinline__ void write_rows(const TreeAttn& P, const TreeItem& it) {
  const int lane = lane_id();
  if (P.n_rows > 0 && it.pg0 == first_page(it.len, P.window) && lane < it.n)
    P.tok[it.t0 + lane] = make_int4(it.row0 + lane, it.n, it.splits, 0);
}

// A sink's share of the normaliser over the maximum M (log2 units). A sink of -inf has
// none, also where there is no key (M = -inf).
__device__ __forceinline__ float sink_term(float sink, float M) {
  return M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sink - M);
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
  // the same for 32 slots from k0 on, bit i: slot k0 + i
  __device__ __forceinline__ uint32_t keys(int k0, int len) const {
    const int off = k0 - len, left = lo - k0;  // first node, first committed key in sight
    const uint64_t nodes = off >= 0 ? (off < 64 ? seen >> off : 0) : (off > -32 ? seen << -off : 0);
    const uint32_t old = off >= 0 ? 0u : off > -32 ? (1u << -off) - 1u : ~0u;
    return (uint32_t)nodes | (old & ~(left <= 0 ? 0u : left < 32 ? (1u << left) - 1u : ~0u));
  }
};
__device__ __forceinline__ Sight sight_of(const TreeAttn& P, const TreeItem& it, const Nodes& nodes, int node) {
  const uint32_t lo = __shfl((uint32_t)nodes.seen, node, 64), hi = __shfl((uint32_t)(nodes.seen >> 32), node, 64);
  const int depth = __shfl(nodes.depth, node, 64);
  Sight s;
  s.lo = P.window > 0 ? it.len + depth - P.window + 1 : 0;
  s.seen = (uint64_t)hi << 32 | lo;
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
  const int g = id % hkv, tile = id / hkv % (unsigned)tiles, item = id / hkv / (unsigned)tiles;
  if (item >= P.n_items) return;  // no barriers below
  TreeItem it;
  if (!find_item(P, item, it)) return;
  const int G = P.hq / P.hkv, cols = it.n * G;
  if (16 * tile >= cols) return;
  const int c = 16 * tile + hl, node = min(c / G, it.n - 1), head = g * G + c % G;
  const bool valid = c < cols;
  const int parent = parent_of(P, it);
  Frag<T> qf[D / 32];
  const T* qb = reinterpret_cast<const T*>(P.q) + ((int64_t)(it.t0 + node) * P.hq + head) * D + 8 * grp;
#pragma unroll
  for (int cc = 0; cc < D / 32; ++cc) qf[cc].load(qb + 32 * cc);
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
  // ids of a block of pages and of those requested ahead of it, lane i: page pg0 + base + i (the split's last past
  // its end); the next block's are loaded a block ahead
  constexpr int BLK = 60;
  const int pages = it.pg1 - it.pg0;
  auto ids_of = [&](int base) { return ptab[it.pg0 + min(base + lane, pages - 1)]; };
  int ids = ids_of(0);
  auto fetch = [&](Page& p, int at) __attribute__((always_inline)) {  // `at`: the page's place in ids
    int pid = __builtin_amdgcn_readlane(ids, at);
    p.ok = pid >= 0 && pid < P.n_pages;
    pid = p.ok ? pid : 0;
    const T* kp = kpool + pid * page_elems + head_off;
    p.vp = vpool + pid * page_elems + head_off;
#pragma unroll
    for (int cc = 0; cc < D / 32; ++cc) p.k[cc].load(kp + (64 * cc + lane) * 8);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) p.v[n].load(p.vp + (64 * n + lane) * 4);
  };
  // four pages in flight, as short contexts are latency alone, the first before the tree's ancestors are worked out:
  // three trees over up to 512 cached tokens, fp32: 6.9 us, 9.9 with one page ahead, 7.4 with eight or with page
  // ids loaded one by one (64 trees over ~3,000: 78, 102 and 85)
  constexpr int PF = 4;
  static_assert(BLK % PF == 0 && BLK + PF <= 64, "a block's ids and those requested ahead of it");
  Page ring[PF];
#pragma unroll
  for (int u = 0; u < PF; ++u) fetch(ring[u], u);
  const Sight sight = sight_of(P, it, nodes_of(P, it, parent), node);
  if (g == 0 && tile == 0) write_rows(P, it);
#pragma unroll
  for (int cc = 0; cc < D / 32; ++cc) qf[cc].keep_if(valid);
  float m = -INFINITY, l = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto attend = [&](Page& cur, int pg) __attribute__((always_inline)) {
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
      if (!cur.ok && lane == 0) set_error(P.err, 1);
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
  };
  for (int base = 0;;) {
    const int next = ids_of(base + BLK), stop = min(pages, base + BLK);
    for (int i = base; i < stop; i += PF) {
#pragma unroll
      for (int u = 0; u < PF; ++u) {
        if (i + u >= stop) break;
        attend(ring[u], it.pg0 + i + u);
        fetch(ring[u], i + u + PF - base);
      }
    }
    if (stop == pages) break;
    base = stop;
    ids = next;
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
    l = l * f + sink_term(sk, M);
  }
  T* o = reinterpret_cast<T*>(P.o) + ((int64_t)(it.t0 + node) * P.hq + head) * D + 4 * grp;
#pragma unroll
  for (int n = 0; n < D / 16; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) Elem<T>::store(o, 16 * n + r, l == 0.f ? 0.f : f * acc[n][r] / l);
}

// ---------------------------------------------------------------------------
// attend, bf16 with head dim 64: 64 columns per wavefront
// ---------------------------------------------------------------------------

// A workgroup of NC wavefronts owns one split of one tree and KV head; each
// wavefront holds NT tiles of 32 columns. The pages go straight to LDS, two
// (32 keys) a step through TRS stages, once for all NC wavefronts. Per step a
// wavefront forms S^T = K Q^T as a 32 x 32 tile per 32 columns and accumulates
// O^T += V^T P^T from it: lane l holds column l % 32 and, with h = l / 32, keys
// 8 q + 4 h + r (element 4 q + r), which is the value product's operand order.
// The scores of step s + 1 are formed beside the weights of step s.
//
// The maximum of a column is raised only when a lane's share of a step's weights
// would pass 2^8, so that most steps have no cross-lane step and no rescale.
//
// Wide trees are bound by no unit alone: 16 trees of 33-64 nodes (7.6 M node and key
// pairs a head) take 192 us with the combine, 650 TFLOP/s. Of its wavefronts' cycles 39%
// have an instruction at work, 34% wait for loads and at barriers, 27% for their turn or
// a result; the matrix cores are busy 30% of the launch, the vector pipe 40%. 18% of the
// wavefronts' steps have no columns (a tree's last column tile), and 992 workgroups on
// 512 places are two uneven rounds. Narrow trees are bound by HBM.
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_void_t;

// O^T tiles of 32 x 32 products: lane l holds column l % 32 and, with h = l / 32, the
// dims (or keys) 8 q + 4 h + r in element 4 q + r.

// keys that are not in sight get a score of -inf; `mine`: the step's keys from the
// lane's first one on
__device__ __forceinline__ void hide(f32x16& t, uint32_t mine) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {  // all ones where the key is in sight: a bit-field extract and a bit select
    const uint32_t in = (uint32_t)((int32_t)(mine << (31 - (8 * (e >> 2) + (e & 3)))) >> 31);
    t[e] = __uint_as_float((in & __float_as_uint(t[e])) | (~in & 0xFF800000u));
  }
}
// a column's largest score of a step, over both of its lanes
__device__ __forceinline__ float largest(const f32x16& t) {
  float m = t[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) m = vmax(m, t[e]);
  const uint32_t u = __float_as_uint(m);
  auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return vmax(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
// weights 2^(score scale - m), rounded to bf16 as the value product takes them (its
// operand type), and their sum after that rounding, so that the quotient is of the
// same weights
__device__ __forceinline__ float weigh(const f32x16& t, float scale_log2, float m, u32x4_t (&pw)[2]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; e += 2) {
    const float p0 = __builtin_amdgcn_exp2f(fmaf(t[e], scale_log2, -m));
    const float p1 = __builtin_amdgcn_exp2f(fmaf(t[e + 1], scale_log2, -m));
    const uint32_t w = pack_bf16(p0, p1);
    pw[e >> 3][(e & 7) >> 1] = w;
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), sum, false);
  }
  return sum;
}
// Value fragments of a step with masked keys: a weight of zero times a value that is
// not finite would not be zero, so such values are set to zero; true for the whole
// wavefront if there were any (add_nonfinite gives them back to the columns that
// see them).
__device__ __forceinline__ bool drop_nonfinite(u32x4_t (&vf)[2][2]) {
  const u16x2_t full = {0x7F80, 0x7F80}, one = {1, 1};
  u16x2_t top = {0, 0};  // the largest exponent field in either half
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, vf[p][dt][i] & 0x7F807F80u));
  const bool odd = top.x == 0x7F80u || top.y == 0x7F80u;
  if (__builtin_amdgcn_ballot_w64(odd) == 0) return false;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // halves times 0 where the exponent is full, else times 1
        const uint32_t w = vf[p][dt][i];
        const u16x2_t keep = __builtin_elementwise_min(full - __builtin_bit_cast(u16x2_t, w & 0x7F807F80u), one);
        vf[p][dt][i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2_t, w) * keep);
      }
  return true;
}
// One lane's column in each of a wavefront's NT tiles: its node and head, what it
// sees, its query, and the running softmax.
constexpr float WEIGHT_LIMIT = 0x1p8f;  // of a lane's 16 weights in a step
template <int NT>
struct Columns {
  int node[NT], head[NT];
  bool valid[NT];
  Sight sight[NT];
  Frag<bf16> qf[NT][4];
  float m_run[NT], m_sub[NT], limit[NT], l[NT];  // limit: -inf until a key is visible
  f32x16 acc[2][NT];                             // [dim tile][column tile]
  bool odd;                                      // values that are not finite were dropped

  // the columns from c0 on, and the loads of their queries
  __device__ __forceinline__ void request(const TreeAttn& P, const TreeItem& it, int g, int c0) {
    const int G = P.hq / P.hkv, lane = lane_id(), fc = lane & 31, h = lane >> 5;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int c = c0 + 32 * j + fc;
      valid[j] = c < it.n * G;
      node[j] = min(c / G, it.n - 1);
      head[j] = g * G + c % G;
      const bf16* qp = reinterpret_cast<const bf16*>(P.q) + ((int64_t)(it.t0 + node[j]) * P.hq + head[j]) * 64 + 8 * h;
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) qf[j][cc].load(qp + 16 * cc);
    }
  }
  __device__ __forceinline__ void start(const TreeAttn& P, const TreeItem& it, int parent) {
    const Nodes nodes = nodes_of(P, it, parent);
    odd = false;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      sight[j] = sight_of(P, it, nodes, node[j]);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) qf[j][cc].keep_if(valid[j]);
      m_run[j] = -INFINITY;
      m_sub[j] = 0.f;
      limit[j] = -INFINITY;
      l[j] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[dt][j][e] = 0.f;
    }
  }
  // S^T of 32 keys
  __device__ __forceinline__ void scores(f32x16 (&t)[NT], const u32x4_t (&kf)[4]) const {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) t[j][e] = 0.f;
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        t[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[cc]),
                                                       __builtin_bit_cast(bf16x8_t, qf[j][cc].v), t[j], 0, 0, 0);
  }
  // hide what a column does not see of the 32 keys from k0 on; `pages`: the keys whose page is there
  __device__ __forceinline__ void mask(f32x16 (&t)[NT], int k0, int len, uint32_t pages) const {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint32_t vis = valid[j] ? sight[j].keys(k0, len) & pages : ~0u;
      hide(t[j], vis >> (4 * (lane_id() >> 5)));
    }
  }
  // tile j's weights of a step, packed, and their sum
  __device__ __forceinline__ float weights(int j, const f32x16& t, float scale_log2, u32x4_t (&pw)[2]) const {
    return weigh(t, scale_log2, m_sub[j], pw);
  }
  // The maximum only has to keep the weights in range, so it is raised when a step's sum says that they are not, and
  // until a column has seen a key; the weights are then formed again.
  __device__ __forceinline__ void raise(int j, const f32x16& t, float scale_log2, u32x4_t (&pw)[2], float& sum) {
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(sum > limit[j]) != 0, 0)) {  // wave-uniform; the empty asm keeps it a branch
      asm volatile("");
      // a column's own lanes decide, so that its bits do not depend on the columns beside it
      const uint32_t o = sum > limit[j];
      auto so = __builtin_amdgcn_permlane32_swap(o, o, false, false);
      const float m_new = (so[0] | so[1]) ? fmaxf(m_run[j], largest(t) * scale_log2) : m_run[j];
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[j] - m_new);
      l[j] *= alpha;
#pragma unroll
      for (int dt = 0; dt < 2; ++dt) acc[dt][j] *= alpha;
      m_run[j] = m_new;
      m_sub[j] = m_new == -INFINITY ? 0.f : m_new;  // masked scores give 2^-inf = 0
      limit[j] = m_new == -INFINITY ? -INFINITY : WEIGHT_LIMIT;
      sum = weights(j, t, scale_log2, pw);
    }
  }
  // O^T += V^T P^T of tile j
  __device__ __forceinline__ void add(int j, const u32x4_t (&vf)[2][2], const u32x4_t (&pw)[2], float sum) {
    l[j] += sum;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int dt = 0; dt < 2; ++dt)
        acc[dt][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf[p][dt]),
                                                             __builtin_bit_cast(bf16x8_t, pw[p]), acc[dt][j], 0, 0, 0);
  }
};
// The steps with masked keys once more, for values that are not finite: added to the
// accumulators of the columns that see them, which makes those infinite or NaN as
// any positive weight does. Steps without masked keys need no such care.
template <int NT>
__device__ __forceinline__ void add_nonfinite(const TreeAttn& P, const TreeItem& it, int g, Columns<NT>& c) {
  constexpr int D = 64;
  const int h = lane_id() >> 5;
  const int32_t* ptab = P.page_table + (int64_t)it.b * P.max_pages;
  for (int pg = it.pg0; pg < it.pg1; ++pg) {
    const int k0 = pg * PAGE, id = uniform(ptab[pg]);
    if (id < 0 || id >= P.n_pages) continue;
    // the pages of steps with masked keys, and at most one page more on either side
    if (k0 + 3 * PAGE <= it.len && !(P.window > 0 && k0 < it.len + it.n - P.window + PAGE) && pg + 2 < it.pg1) {
      const int before = uniform(ptab[max(pg - 1, it.pg0)]), after = uniform(ptab[pg + 1]);
      if (before >= 0 && before < P.n_pages && after >= 0 && after < P.n_pages) continue;
    }
    const bf16* page = reinterpret_cast<const bf16*>(P.v_pool) + ((int64_t)id * P.hkv + g) * PAGE * D;
    for (int slot = 0; slot < PAGE; ++slot)
#pragma unroll
      for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint16_t bits = page[v_off(slot, 32 * dt + 8 * (e >> 2) + 4 * h + (e & 3))].bits;
          const bool bad = (bits & 0x7F80u) == 0x7F80u;
#pragma unroll
          for (int j = 0; j < NT; ++j)
            c.acc[dt][j][e] += bad & c.valid[j] & c.sight[j].key(k0 + slot, it.len, it.n) ? bf16_to_f32(bits) : 0.f;
        }
  }
}
// the lane's dims of each column: a partial row, or o with the sink
template <int NT>
__device__ __forceinline__ void finish(const TreeAttn& P, const TreeItem& it, const Columns<NT>& c) {
  constexpr int D = 64;
  const int h = lane_id() >> 5;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const uint32_t u = __float_as_uint(c.l[j]);
    auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    float l_tot = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (!c.valid[j]) continue;
    if (it.splits > 1) {
      const int64_t row = (int64_t)(it.row0 + c.node[j]) * P.hq + c.head[j];
      if (h == 0) *reinterpret_cast<float2*>(P.part_ml + 2 * row) = make_float2(c.m_run[j], l_tot);
#pragma unroll
      for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(P.part_acc + row * D + 32 * dt + 8 * q + 4 * h) =
              make_float4(c.acc[dt][j][4 * q], c.acc[dt][j][4 * q + 1], c.acc[dt][j][4 * q + 2], c.acc[dt][j][4 * q + 3]);
      continue;
    }
    float f = 1.0f;
    if (P.sinks) {
      const float sk = P.sinks[c.head[j]] * LOG2E, M = fmaxf(c.m_run[j], sk);
      f = c.m_run[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(c.m_run[j] - M);
      l_tot = l_tot * f + sink_term(sk, M);
    }
    const float inv = l_tot == 0.f ? 0.f : f / l_tot;
    // the lanes of a column trade halves, so that each writes eight dims at a time
    bf16* o = reinterpret_cast<bf16*>(P.o) + ((int64_t)(it.t0 + c.node[j]) * P.hq + c.head[j]) * D + 8 * h;
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        uint32_t w[2][2];  // [q][pair of dims]
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int e = 4 * (q + k) + 2 * r;
            w[k][r] = pack_bf16(c.acc[dt][j][e] * inv, c.acc[dt][j][e + 1] * inv);
          }
        auto lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
        auto hi = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
        *reinterpret_cast<u32x4_t*>(o + 32 * dt + 8 * q) = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
      }
  }
}

// A stage holds K of a step's two pages, then V of both, as in the pool but for the
// 16-byte chunks of V: 128-byte block b of a 512-byte dim tile sits at b ^ (tile & 1),
// so that the lanes of a half tile read all banks.
constexpr uint32_t STAGE_PAGE = 2 * PAGE * 64;  // bytes of K (or V) of a page of one KV head
// a step's key fragments: key l % 32 (page l / 16 % 2), dims 8 h .. of a 16-dim chunk
__device__ __forceinline__ void stage_keys(u32x4_t (&kf)[4], const uint8_t* stg) {
  const int fc = lane_id() & 31, h = lane_id() >> 5;
  const uint32_t ko = (fc >> 4) * STAGE_PAGE + ((h * 16 + (fc & 15)) * 16);
#pragma unroll
  for (int cc = 0; cc < 4; ++cc) kf[cc] = *reinterpret_cast<const u32x4_t*>(stg + ko + 512 * cc);
}
// The softmax and the value products of the step at page pg from its scores `sc` and
// its stage, and the scores `sn` of the next step from the stage behind it; ok: its
// pages are there.
template <int NT>
__device__ __forceinline__ void attend_stage(const TreeAttn& P, const TreeItem& it, Columns<NT>& col, f32x16 (&sc)[NT],
                                             f32x16 (&sn)[NT], const uint8_t* stg, const uint8_t* nxt, int pg,
                                             const bool (&ok)[2]) {
  const int lane = lane_id(), fc = lane & 31, h = lane >> 5;
  u32x4_t kf[4];
  stage_keys(kf, nxt);
  const int k0 = pg * PAGE;
  const bool second = pg + 1 < it.pg1;
  const bool edge = k0 + 2 * PAGE > it.len || (P.window > 0 && k0 < it.len + it.n - P.window) || !ok[0] || !ok[1] || !second;
  if (__builtin_expect(edge, 0)) {  // wave-uniform; the empty asm keeps it a branch
    asm volatile("");
    if ((!ok[0] || (!ok[1] && second)) && lane == 0) set_error(P.err, 1);
    col.mask(sc, k0, it.len, (ok[0] ? 0xFFFFu : 0u) | (ok[1] && second ? 0xFFFF0000u : 0u));
  }
  // dim l % 32 of a tile of 32, value rows 4 h .. and 8 + 4 h ..
  const uint32_t vbase = (fc >> 4) * 512 + (fc & 15) * 8 + (((uint32_t)h ^ ((fc >> 4) & 1)) << 7);
  u32x4_t vf[2][2];  // [page][dim tile]
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int dt = 0; dt < 2; ++dt) {
      const uint8_t* v = stg + (2 + p) * STAGE_PAGE + 1024 * dt + vbase;
      const u32x2_t a = *reinterpret_cast<const u32x2_t*>(v), c = *reinterpret_cast<const u32x2_t*>(v + 256);
      vf[p][dt] = __builtin_shufflevector(a, c, 0, 1, 2, 3);
    }
  u32x4_t pw[NT][2];  // [column tile][page]: the weights, packed
  float sum[NT];
  // the next scores' products among the vector instructions of the first tile's weights, the first tile's value
  // products among those of the second's (24 trees of 16-32: 140 us, 146 with all weights before all value products)
  __builtin_amdgcn_sched_barrier(0);
  col.scores(sn, kf);
  sum[0] = col.weights(0, sc[0], P.scale_log2, pw[0]);
#pragma unroll
  for (int i = 0; i < 4 * NT; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x402, NT == 2 ? 6 : 12, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  }
  col.raise(0, sc[0], P.scale_log2, pw[0], sum[0]);
  if (__builtin_expect(edge, 0)) {
    asm volatile("");
    col.odd |= drop_nonfinite(vf);
  }
  if constexpr (NT == 2) {
    __builtin_amdgcn_sched_barrier(0);
    col.add(0, vf, pw[0], sum[0]);
    sum[1] = col.weights(1, sc[1], P.scale_log2, pw[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 12, 0);
    }
    col.raise(1, sc[1], P.scale_log2, pw[1], sum[1]);
  }
  col.add(NT - 1, vf, pw[NT - 1], sum[NT - 1]);
}
// Piece w of a step, 1 KB, into its stage: half w % 2 of K of page 0, K of page 1, V
// of page 0, V of page 1 (w / 2) of pool page `id`; a `range` of 0 touches no memory.
template <int POLICY>
__device__ __forceinline__ void load_piece(const TreeAttn& P, uint8_t* stg, int w, int g, int id, int range) {
  const int lane = lane_id();
  const uint8_t* pool = reinterpret_cast<const uint8_t*>(w < 4 ? P.k_pool : P.v_pool) + (int64_t)g * STAGE_PAGE;
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(pool) + id * ((int64_t)P.hkv * STAGE_PAGE), 0, range, 0x00020000);
  const uint32_t at = 1024u * (w & 1) + 16u * lane;
  const uint32_t vo = w < 4 ? at : at ^ (((at >> 9) & 1u) << 7);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t)(stg + 1024 * w), 16, vo, 0, 0, POLICY);
}
// Hands the stages over: this wavefront's reads of LDS have returned (lgkmcnt), all
// its loads but the last N have landed, and the empty asm keeps LDS accesses on their
// side of the barrier.
template <int N>
__device__ __forceinline__ void publish_stages() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (N >> 4 << 14));  // vmcnt(N) expcnt(7) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int NC, int NT, int TRS>
__global__ __launch_bounds__(64 * NC, NT == 1 ? 4 : 2) void tree_attn_wide_kernel(TreeAttn P, int tiles) {
  constexpr uint32_t PB = STAGE_PAGE;
  constexpr int LD = 8 / NC;                         // 1 KB loads per wavefront and step
  // where one workgroup takes all columns of a step whose pages no cache holds: the streaming policy (3% at 48
  // trees of 8-16 nodes)
  constexpr int POLICY = NC == 2 ? 2 : 0;
  static_assert(TRS % 2 == 0 && TRS <= 6 && 8 % NC == 0, "stages alternate between two score sets");
  __shared__ __align__(1024) uint8_t s0[4 * PB];
  __shared__ __align__(1024) uint8_t s1[4 * PB];
  __shared__ __align__(1024) uint8_t s2[4 * PB];
  __shared__ __align__(1024) uint8_t s3[4 * PB];
  __shared__ __align__(1024) uint8_t s4[4 * PB];
  __shared__ __align__(1024) uint8_t s5[4 * PB];
  auto stage_of = [&](int s) __attribute__((always_inline)) {
    return s == 0 ? s0 : s == 1 ? s1 : s == 2 ? s2 : s == 3 ? s3 : s == 4 ? s4 : s5;
  };
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  // workgroups are dealt to the eight XCDs in turn: the column tiles of one split and head go to the same one
  const unsigned hkv = P.hkv, slot = blockIdx.x >> 3;
  const unsigned pair = slot / (unsigned)tiles * 8 + (blockIdx.x & 7);
  const int tile = slot % (unsigned)tiles, g = pair % hkv, item = pair / hkv;
  if (item >= P.n_items) return;
  TreeItem it;
  if (!find_item(P, item, it)) return;  // uniform over the workgroup
  const int G = P.hq / P.hkv, cols = it.n * G;
  if (32 * NT * NC * tile >= cols) return;
  const int c0 = 32 * NT * (NC * tile + wave);
  const bool busy = c0 < cols;  // wave-uniform; a wavefront without columns only loads
  const int32_t* ptab = P.page_table + (int64_t)it.b * P.max_pages;
  const int n_steps = (it.pg1 - it.pg0 + 1) / 2;

  // page ids of steps base .. base + 31, lane i: page pg0 + 2 base + i (the split's last page past its end). A
  // block of IDB steps and the requests ahead of it find their ids in one register; the next block's are
  // loaded a block ahead.
  constexpr int IDB = 24;
  static_assert(IDB % TRS == 0 && IDB + TRS - 1 <= 32, "a block's ids and those requested ahead of it");
  auto ids_of = [&](int base) __attribute__((always_inline)) {
    return ptab[min(it.pg0 + 2 * base + lane, it.pg1 - 1)];
  };
  int ids = ids_of(0), base = 0;
  const int parent = parent_of(P, it);

  Columns<NT> col;
  col.request(P, it, g, c0);

  auto page_of = [&](int step, int which, bool& good) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, 2 * (step - base) + which);
    good = id >= 0 && id < P.n_pages;
    return good ? id : 0;
  };
  // request a step's pages; past the split's end the loads have no range, so that every step counts the same number
  // of them
  auto request = [&](uint8_t* stg, int step) __attribute__((always_inline)) {
    const int range = step < n_steps ? PB : 0;
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int w = wave * LD + u;
      bool good;
      const int id = page_of(step, (w >> 1) & 1, good);
      load_piece<POLICY>(P, stg, w, g, id, range);
    }
  };

  // the first pages before the tree's ancestors are worked out: one round of memory less in front of the first step
#pragma unroll
  for (int s = 0; s < TRS - 1; ++s) {
    request(stage_of(s), s);
    __builtin_amdgcn_sched_barrier(0);
  }
  col.start(P, it, parent);

  // Step s sits in stage s % TRS. In step s its scores are there already; step s + TRS - 1 is requested into the
  // stage step s - 1 left, the scores of step s + 1 are formed, and before the barrier a wavefront waits for its
  // loads of step s + 2.
  auto publish = [&]() __attribute__((always_inline)) { publish_stages<LD * (TRS - 3)>(); };
  publish();
  f32x16 sc[2][NT];
  if (busy) {
    u32x4_t kf[4];
    stage_keys(kf, s0);
    col.scores(sc[0], kf);
  }
  auto one = [&](auto U_, int step) __attribute__((always_inline)) {
    constexpr int U = decltype(U_)::value;
    if (step < n_steps) {  // uniform
      request(stage_of((U + TRS - 1) % TRS), step + TRS - 1);
      if (busy) {
        bool ok[2];
        page_of(step, 0, ok[0]);
        page_of(step, 1, ok[1]);
        attend_stage<NT>(P, it, col, sc[U % 2], sc[(U + 1) % 2], stage_of(U), stage_of((U + 1) % TRS), it.pg0 + 2 * step, ok);
      }
    }
    publish();
  };
  while (true) {
    const int ids_next = ids_of(base + IDB), stop = min(n_steps, base + IDB);
    for (int step = base; step < stop; step += TRS) {
      one(std::integral_constant<int, 0>{}, step);
      one(std::integral_constant<int, 1>{}, step + 1);
      one(std::integral_constant<int, 2>{}, step + 2);
      one(std::integral_constant<int, 3>{}, step + 3);
      if constexpr (TRS > 4) {
        one(std::integral_constant<int, 4>{}, step + 4);
        one(std::integral_constant<int, 5>{}, step + 5);
      }
    }
    if (stop == n_steps) break;
    base = stop;
    ids = ids_next;
  }
  __builtin_amdgcn_s_waitcnt(0);  // no load into LDS may outlive the workgroup

  if (g == 0 && tile == 0 && wave == 0) write_rows(P, it);
  if (col.odd) add_nonfinite<NT>(P, it, g, col);
  finish<NT>(P, it, col);
}

// The same products for few columns: one wavefront per split, KV head and 32 columns,
// its pages straight to registers, two steps in flight. Nothing is shared,
// so there is no LDS and no barrier, and the wavefronts of a SIMD hide each other's
// loads and products. Bound by HBM on large batches (48 trees of 1-4 nodes behind 4-16 K
// tokens: 102 us, 5.7 TB/s), by the latency of row offsets, page ids and pages one
// after the other on small ones (one tree of 4 behind 6 K: 8.9 us).
template <bool STREAM>
__global__ __launch_bounds__(64, 3) void tree_attn_narrow_kernel(TreeAttn P, int tiles) {
  constexpr int D = 64, PE = PAGE * D;
  const int lane = lane_id();
  const unsigned hkv = P.hkv, slot = blockIdx.x >> 3;
  const unsigned pair = slot / (unsigned)tiles * 8 + (blockIdx.x & 7);
  const int tile = slot % (unsigned)tiles, g = pair % hkv, item = pair / hkv;
  if (item >= P.n_items) return;
  TreeItem it;
  if (!find_item(P, item, it)) return;
  const int G = P.hq / P.hkv, cols = it.n * G, c0 = 32 * tile;
  if (c0 >= cols) return;
  const int32_t* ptab = P.page_table + (int64_t)it.b * P.max_pages;
  const int n_steps = (it.pg1 - it.pg0 + 1) / 2;
  const int64_t page_elems = (int64_t)P.hkv * PE;
  const bf16* kpool = reinterpret_cast<const bf16*>(P.k_pool) + (int64_t)g * PE;
  const bf16* vpool = reinterpret_cast<const bf16*>(P.v_pool) + (int64_t)g * PE;
  const int fc = lane & 31, h = lane >> 5;

  // page ids of steps base .. base + 31, lane i: page pg0 + 2 base + i
  auto ids_of = [&](int base) __attribute__((always_inline)) {
    return ptab[min(it.pg0 + 2 * base + lane, it.pg1 - 1)];
  };
  int ids = ids_of(0);
  struct Step {
    u32x4_t k[4];     // key fc of the step, dims 8 h .. of each 16-dim chunk
    u32x2_t v[2][4];  // [page][2 dim tile + half]: dim fc of a tile of 32, value rows 4 h .. and 8 + 4 h ..
    bool ok[2];
  };
  const uint32_t ko = (h * 16 + (fc & 15)) * 8, vo = (fc >> 4) * 256 + (fc & 15) * 4 + h * 64;
  auto fetch = [&](Step& st, int step, int at) __attribute__((always_inline)) {  // `at`: the step's place in ids
    int64_t off[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int id = __builtin_amdgcn_readlane(ids, 2 * at + p);
      const bool good = id >= 0 && id < P.n_pages;
      st.ok[p] = good && it.pg0 + 2 * step + p < it.pg1;
      off[p] = (good ? id : 0) * page_elems;
    }
    const bf16* kp = kpool + (fc < 16 ? off[0] : off[1]) + ko;
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) st.k[cc] = STREAM ? ld_stream16(kp + 256 * cc) : *reinterpret_cast<const u32x4_t*>(kp + 256 * cc);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16* vp = vpool + off[p] + vo + 512 * (i >> 1) + 128 * (i & 1);
        st.v[p][i] = STREAM ? ld_stream8(vp) : *reinterpret_cast<const u32x2_t*>(vp);
      }
  };

  const int parent = parent_of(P, it);
  Columns<1> col;
  col.request(P, it, g, c0);
  Step a, b;
  fetch(a, 0, 0);
  fetch(b, 1, 1);
  col.start(P, it, parent);
  auto attend = [&](Step& st, int step) __attribute__((always_inline)) {
    f32x16 sc[1];
    col.scores(sc, st.k);
    const int pg = it.pg0 + 2 * step, k0 = pg * PAGE;
    const bool edge = k0 + 2 * PAGE > it.len || (P.window > 0 && k0 < it.len + it.n - P.window) || !st.ok[0] || !st.ok[1];
    if (__builtin_expect(edge, 0)) {
      asm volatile("");
      if ((!st.ok[0] || (!st.ok[1] && pg + 1 < it.pg1)) && lane == 0) set_error(P.err, 1);
      col.mask(sc, k0, it.len, (st.ok[0] ? 0xFFFFu : 0u) | (st.ok[1] ? 0xFFFF0000u : 0u));
    }
    u32x4_t pw[2];
    float sum = col.weights(0, sc[0], P.scale_log2, pw);
    col.raise(0, sc[0], P.scale_log2, pw, sum);
    u32x4_t vf[2][2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int dt = 0; dt < 2; ++dt) vf[p][dt] = __builtin_shufflevector(st.v[p][2 * dt], st.v[p][2 * dt + 1], 0, 1, 2, 3);
    if (__builtin_expect(edge, 0)) {
      asm volatile("");
      col.odd |= drop_nonfinite(vf);
    }
    col.add(0, vf, pw, sum);
  };
  // blocks of 30 steps, whose ids and those of the two steps requested ahead sit in one register; a step past
  // the end reads the last page again and is masked
  constexpr int BLK = 30;
  for (int base = 0;;) {
    const int next = ids_of(base + BLK), stop = min(n_steps, base + BLK);
    int step = base;
    for (; step + 1 < stop; step += 2) {
      attend(a, step);
      fetch(a, step + 2, step + 2 - base);
      attend(b, step + 1);
      fetch(b, step + 3, step + 3 - base);
    }
    if (step < stop) attend(a, step);  // an odd number of steps: only at the split's end
    if (stop == n_steps) break;
    base = stop;
    ids = next;
  }
  if (g == 0 && tile == 0) write_rows(P, it);
  if (col.odd) add_nonfinite<1>(P, it, g, col);
  finish<1>(P, it, col);
}

// The kernel for a step and the columns that one of its wavefronts or workgroups
// takes. bf16 with head dim 64 has the 32 x 32 products; their loads need 16-byte
// aligned pools. `cols` is the largest tree's node and head pairs per KV head; `few`:
// the step's pages fit the caches and its splits leave compute units idle; `one_each`:
// no tree is split. Latency bounds such steps, and bandwidth or the vector pipe the
// rest. Streaming loads serve pages that one wavefront or workgroup reads, once; with
// several column tiles they make each fetch its pages anew. Measured in us by events
// around the launch, 64 query heads on 8 KV heads, six sets of pools in turn, contexts
// of 4-16 K tokens unless given (one draw of the sizes for all forms, not the one of the
// figures at the kernels: the 16 wide trees here have 5.3 M pairs). NARROW2 was
// NARROW_STREAM with two column tiles a wavefront, measured on an earlier build.
//   up to 32 columns, 256 windowed trees of 1-4 nodes: NARROW_STREAM 18.5, NARROW 21.8; 48 trees of 1-4
//     NARROW_STREAM 102, NARROW 114, WIDE2 108; one tree of 4 behind 6 K NARROW 9.0, WIDE1 9.8
//   few or one each, up to 96: 256 windowed trees of 2-12 NARROW 32.3, NARROW_STREAM 33.8, WIDE2 34.8, WIDE1 36.2;
//     one tree of 8 behind 6 K NARROW 9.9, WIDE1 10.3
//   few or one each, above: 256 windowed trees of 8-16 WIDE1 40.8, WIDE2 41.7, NARROW 45; one tree of 16 behind 6 K
//     WIDE1 11.9, NARROW 12.1, WIDE2 14.0, of 64 WIDE1 21.6, NARROW 22.3, WIDE4 23.4; 16 windowed trees of 17-30
//     WIDE1 11.0, NARROW 11.4, WIDE4 14.6
//   up to 128, 48 trees of 1-8: WIDE2 109 + 5 for the combine, NARROW2 108 + 9, NARROW 156; 128 trees of 1-8 WIDE2
//     308 + 6, NARROW2 303 + 13; 24 trees of 1-8 WIDE2 49 + 6, NARROW2 53 + 8, NARROW 56; 48 trees of 8-16 WIDE1
//     122-125 + 16, WIDE2 124-129 + 8, WIDE4 154-159 + 8
//   above, 24 trees of 16-32: WIDE4 139 + 7, WIDE1 135-145 + 9, WIDE2 153-156 + 7; 16 of 33-64 behind 8-16 K WIDE4
//     163-167 + 7, WIDE1 160-163 + 9, WIDE2 187-193 + 7; one workgroup of eight wavefronts for 512 columns was 10-20%
//     slower than two of WIDE4, whose barriers stop fewer wavefronts
TreeForm tree_attn_form(int dtype, int head_dim, const void* k_pool, const void* v_pool, int cols, bool few, bool one_each) {
  if (dtype != 1 || head_dim != 64 || ((uintptr_t)k_pool | (uintptr_t)v_pool) % 16) return {TREE_ANY, 16, 12};
  if (cols <= 32) return {few ? TREE_NARROW : TREE_NARROW_STREAM, 32, 8};
  if (few || one_each) return cols <= 96 ? TreeForm{TREE_NARROW, 32, 8} : TreeForm{TREE_WIDE1, 128, 3};
  return cols <= 128 ? TreeForm{TREE_WIDE2, 128, 4} : TreeForm{TREE_WIDE4, 256, 2};
}

hipError_t launch_tree_attn(int dtype, int head_dim, const TreeAttn& p, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  const int cols = p.max_nodes * (p.hq / p.hkv), tiles = (cols + p.form.cols - 1) / p.form.cols;
  // groups in multiples of eight: one for each XCD
  const int64_t groups = ((int64_t)p.n_items * p.hkv + 7) / 8 * 8 * tiles;
  if (groups > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 grid((unsigned)groups);
  switch (p.form.kind) {
    case TREE_NARROW: hipLaunchKernelGGL((tree_attn_narrow_kernel<false>), grid, dim3(64), 0, s, p, tiles); break;
    case TREE_NARROW_STREAM: hipLaunchKernelGGL((tree_attn_narrow_kernel<true>), grid, dim3(64), 0, s, p, tiles); break;
    case TREE_WIDE1: hipLaunchKernelGGL((tree_attn_wide_kernel<4, 1, 6>), grid, dim3(256), 0, s, p, tiles); break;
    case TREE_WIDE2: hipLaunchKernelGGL((tree_attn_wide_kernel<2, 2, 4>), grid, dim3(128), 0, s, p, tiles); break;
    case TREE_WIDE4: hipLaunchKernelGGL((tree_attn_wide_kernel<4, 2, 6>), grid, dim3(256), 0, s, p, tiles); break;
    default: {
      const dim3 fours((unsigned)((groups + 3) / 4)), block(256);
      if (dtype == 0) {
        if (head_dim == 32) hipLaunchKernelGGL((tree_attn_kernel<float, 32>), fours, block, 0, s, p, tiles);
        else hipLaunchKernelGGL((tree_attn_kernel<float, 64>), fours, block, 0, s, p, tiles);
      } else {
        if (head_dim == 32) hipLaunchKernelGGL((tree_attn_kernel<bf16, 32>), fours, block, 0, s, p, tiles);
        else hipLaunchKernelGGL((tree_attn_kernel<bf16, 64>), fours, block, 0, s, p, tiles);
      }
    }
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// combine: o_h = sum_s 2^(m_s - M) acc_s / (2^(sink_h log2e - M) + sum_s 2^(m_s - M) l_s)
// ---------------------------------------------------------------------------

// D / 4 lanes per partial row of a (node, head) of the trees with several splits: a
// lane group per pair, which goes through its splits four at a time, or, with many
// splits or few pairs (MANY), the whole wavefront, its lane groups joined at the end.
// Bound by three rounds of latency, then by HBM: 31 splits of one tree 4.8 us (MANY); up
// to four splits of 16 trees of 33-64 nodes, 20 MB of rows, 7.4 us (MANY 12.2, more than
// half of it vector work of the joins), up to six, 52 MB, 11 us; 48 trees of 1-8 5.5 (MANY 5.1).
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeCombine P) {
  constexpr int LR = D / 4, RW = 64 / LR, STEP = MANY ? RW : 1;
  const int lane = lane_id(), sub = lane / LR, dim = 4 * (lane % LR);
  const unsigned wave = blockIdx.x * 4 + uniform(threadIdx.x >> 6), id = MANY ? wave : wave * RW + sub, hq = P.hq;
  const int t = id / hq, h = id % hq;
  if (t >= P.n_tokens) return;
  const int4 tok = P.tok[t];
  const int row0 = tok.x, n = tok.y, splits = MANY ? uniform(tok.z) : tok.z;
  // rows without splits, and rows of no tree
  if (splits <= 1 || row0 < 0 || n <= 0 || n > TREE_MAX_NODES || (int64_t)row0 + (int64_t)(splits - 1) * n >= P.n_rows) return;
  const float sink = P.sinks ? P.sinks[h] * LOG2E : 0.f;
  float M = -INFINITY, L = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  // U rows in flight per lane
  auto join = [&](auto U_) __attribute__((always_inline)) {
    constexpr int U = decltype(U_)::value;
    for (int k0 = MANY ? sub : 0; k0 < splits; k0 += U * STEP) {
      float2 ml[U];
      float4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {  // past the end: the last split again, with no weight
        const int k = k0 + u * STEP;
        const int64_t row = (int64_t)(row0 + min(k, splits - 1) * n) * P.hq + h;
        ml[u] = *reinterpret_cast<const float2*>(P.part_ml + 2 * row);
        v[u] = *reinterpret_cast<const float4*>(P.part_acc + row * D + dim);
        ml[u].x = k < splits ? ml[u].x : -INFINITY;
      }
      float Mn = M;
#pragma unroll
      for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, ml[u].x);
      const float base = Mn == -INFINITY ? 0.f : Mn, r = __builtin_amdgcn_exp2f(M - base);
      L *= r;
      a.x *= r; a.y *= r; a.z *= r; a.w *= r;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = k0 + u * STEP < splits;  // a row that is not finite keeps its weight
        const float f = in ? __builtin_amdgcn_exp2f(ml[u].x - base) : 0.f;
        L += in ? ml[u].y * f : 0.f;
        a.x += in ? v[u].x * f : 0.f; a.y += in ? v[u].y * f : 0.f;
        a.z += in ? v[u].z * f : 0.f; a.w += in ? v[u].w * f : 0.f;
      }
      M = Mn;
    }
  };
  if (!MANY) join(std::integral_constant<int, 4>{});
  else if (splits <= 2 * RW) join(std::integral_constant<int, 2>{});
  else join(std::integral_constant<int, 8>{});
  // join the lane groups, then the sink
  float Mt = M;
  if (MANY)
#pragma unroll
    for (int o = LR; o < 64; o <<= 1) Mt = fmaxf(Mt, __shfl_xor(Mt, o, 64));
  if (P.sinks) Mt = fmaxf(Mt, sink);
  const float f = __builtin_amdgcn_exp2f(M - (Mt == -INFINITY ? 0.f : Mt));
  L *= f;
  a.x *= f; a.y *= f; a.z *= f; a.w *= f;
  if (MANY)
#pragma unroll
    for (int o = LR; o < 64; o <<= 1) {
      L += __shfl_xor(L, o, 64);
      a.x += __shfl_xor(a.x, o, 64);
      a.y += __shfl_xor(a.y, o, 64);
      a.z += __shfl_xor(a.z, o, 64);
      a.w += __shfl_xor(a.w, o, 64);
    }
  if (P.sinks) L += sink_term(sink, Mt);
  if (MANY && sub != 0) return;
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  store4(reinterpret_cast<T*>(P.o) + ((int64_t)t * P.hq + h) * D + dim,
         make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
}

template <typename T, int D>
static void combine_impl(const TreeCombine& p, hipStream_t s) {
  const int64_t pairs = (int64_t)p.n_tokens * p.hq;
  constexpr int per_block = 4 * (256 / D);  // a lane group each
  // eight splits in two rounds of loads; pairs for up to two rounds of wavefronts on the whole GPU
  if (p.max_splits > 8 || pairs <= 16384) hipLaunchKernelGGL((tree_combine_kernel<T, D, true>), dim3((unsigned)((pairs + 3) / 4)), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((tree_combine_kernel<T, D, false>), dim3((unsigned)((pairs + per_block - 1) / per_block)), dim3(256), 0, s, p);
}

hipError_t launch_tree_combine(int dtype, int head_dim, const TreeCombine& p, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  if ((int64_t)p.n_tokens * p.hq > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (dtype == 0) head_dim == 32 ? combine_impl<float, 32>(p, s) : combine_impl<float, 64>(p, s);
  else head_dim == 32 ? combine_impl<bf16, 32>(p, s) : combine_impl<bf16, 64>(p, s);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// accept
// ---------------------------------------------------------------------------

// One wavefront per tree, lane i = node i. From the root (node 0) the walk goes to
// the lowest child whose drafted id equals the draw at its parent: one ballot per
// step, at most 64 steps (a child comes after its parent). Bound by latency: two
// rounds of loads and the walk, 512 trees of 1-64 nodes 4.6 us.
__global__ __launch_bounds__(64) void tree_accept_kernel(TreeAccept P) {
  const int b = blockIdx.x, lane = lane_id();
  const int t0 = P.cu_q[b], n = P.cu_q[b + 1] - t0;
  int count = 0, last = -1;
  if (n < 0 || n > TREE_MAX_NODES || t0 < 0 || t0 > P.n_tokens - n) {
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
