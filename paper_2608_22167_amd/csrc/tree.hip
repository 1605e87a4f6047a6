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
#include <type_traits>

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

// ---------------------------------------------------------------------------
// attend, bf16 with head dim 64: 64 columns per wavefront
// ---------------------------------------------------------------------------

// A workgroup of NC wavefronts owns one split of one tree and KV head; each
// wavefront holds 64 columns, two tiles of 32. The pages go straight to LDS, two
// (32 keys) a step through TRS stages, once for all NC wavefronts. Per step a
// wavefront forms S^T = K Q^T as a 32 x 32 tile per 32 columns and accumulates
// O^T += V^T P^T from it: lane l holds column l % 32 and, with h = l / 32, keys
// 8 q + 4 h + r (element 4 q + r), which is the value product's operand order.
// The scores of step s + 1 are formed beside the weights of step s.
//
// The maximum of a column is raised only when a lane's share of a step's weights
// would pass 2^8, so that most steps have no cross-lane step and no rescale.
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_void_t;

template <int NC, int TRS>
__global__ __launch_bounds__(64 * NC, 2) void tree_attn_wide_kernel(TreeAttn P, int tiles) {
  constexpr int D = 64, PE = PAGE * D, PB = 2 * PE;  // elements and bytes of a page of one KV head
  constexpr int LD = 8 / NC;                         // 1 KB loads per wavefront and step
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
  const unsigned hkv = P.hkv;
  const int g = blockIdx.x % hkv, tile = blockIdx.x / hkv % (unsigned)tiles, item = blockIdx.x / hkv / (unsigned)tiles;
  TreeItem it;
  if (!load_item(P, item, it)) return;
  const int G = P.hq / P.hkv, cols = it.n * G;
  if (64 * NC * tile >= cols) return;
  const int c0 = 64 * (NC * tile + wave);
  const bool busy = c0 < cols;  // wave-uniform; a wavefront without columns only loads
  const int32_t* ptab = P.page_table + (int64_t)it.b * P.max_pages;
  const int n_steps = (it.pg1 - it.pg0 + 1) / 2;

  // this lane's column in each of the wavefront's two tiles
  const int fc = lane & 31, h = lane >> 5;
  int node[2], head[2];
  bool valid[2];
  Sight sight[2];
  Frag<bf16> qf[2][4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = c0 + 32 * j + fc;
    valid[j] = c < cols;
    node[j] = min(c / G, it.n - 1);
    head[j] = g * G + c % G;
    sight[j] = sight_of(P, it, node[j]);
    const bf16* qp = reinterpret_cast<const bf16*>(P.q) + ((int64_t)(it.t0 + node[j]) * P.hq + head[j]) * D + 8 * h;
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) {
      qf[j][cc].load(qp + 16 * cc);
      qf[j][cc].keep_if(valid[j]);
    }
  }

  // page ids of steps base .. base + 31, lane i: page pg0 + 2 base + i (the split's last page past its end). A
  // block of IDB steps and the requests ahead of it find their ids in one register; the next block's are
  // loaded a block ahead.
  constexpr int IDB = 24;
  static_assert(IDB % TRS == 0 && IDB + TRS - 1 <= 32, "a block's ids and those requested ahead of it");
  auto ids_of = [&](int base) __attribute__((always_inline)) {
    return ptab[min(it.pg0 + 2 * base + lane, it.pg1 - 1)];
  };
  int ids = ids_of(0), base = 0;
  const int64_t page_bytes = (int64_t)P.hkv * PB;
  // piece w of a step, 1 KB: half w % 2 of K of page 0, K of page 1, V of page 0, V of page 1 (w / 2). The 16-byte
  // chunks of V are permuted on the way (128-byte block b of a 512-byte dim tile to b ^ (tile & 1)), so that the
  // lanes of a half tile read all banks.
  auto page_of = [&](int step, int which, bool& good) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, 2 * (step - base) + which);
    good = id >= 0 && id < P.n_pages;
    return good ? id : 0;
  };
  auto request = [&](uint8_t* stg, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int w = wave * LD + u;
      bool good;
      const int id = page_of(step, (w >> 1) & 1, good);
      const uint8_t* pool = reinterpret_cast<const uint8_t*>(w < 4 ? P.k_pool : P.v_pool) + (int64_t)g * PB;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(pool) + id * page_bytes, 0, PB, 0x00020000);
      const uint32_t at = 1024u * (w & 1) + 16u * lane;
      const uint32_t vo = w < 4 ? at : at ^ (((at >> 9) & 1u) << 7);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t)(stg + 1024 * w), 16, vo, 0, 0, 0);
    }
  };

  constexpr float WEIGHT_LIMIT = 0x1p8f;       // of a lane's 16 weights in a step
  float m_run[2], m_sub[2], limit[2], l[2];    // limit: -inf until a key is visible
  f32x16 acc[2][2];                            // [dim tile][column tile]
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    m_run[j] = -INFINITY;
    m_sub[j] = 0.f;
    limit[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[dt][j][e] = 0.f;
  }
  // fragment addresses: key fc of the step (page fc / 16), dims 8 h .. of a 16-dim chunk; dim fc of a tile of 32,
  // value rows 4 h .. and 8 + 4 h ..
  const uint32_t ko = (fc >> 4) * PB + ((h * 16 + (fc & 15)) * 16);
  const uint32_t vbase = (fc >> 4) * 512 + (fc & 15) * 8 + (((uint32_t)h ^ ((fc >> 4) & 1)) << 7);

  struct Scores {
    f32x16 t[2];
  };
  auto load_keys = [&](u32x4_t (&kf)[4], const uint8_t* stg) __attribute__((always_inline)) {
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) kf[cc] = *reinterpret_cast<const u32x4_t*>(stg + ko + 512 * cc);
  };
  auto scores = [&](Scores& sc, const u32x4_t (&kf)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc.t[j][e] = 0.f;
#pragma unroll
    for (int cc = 0; cc < 4; ++cc)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        sc.t[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[cc]),
                                                          __builtin_bit_cast(bf16x8_t, qf[j][cc].v), sc.t[j], 0, 0, 0);
  };
  // the keys of a step that a column sees, bit i: key i
  auto visible = [&](int j, int k0, uint32_t pages) __attribute__((always_inline)) {
    const int off = k0 - it.len, lo = sight[j].lo - k0;  // first node, first committed key in sight
    const uint64_t nodes = off >= 0 ? (off < 64 ? sight[j].seen >> off : 0) : (off > -32 ? sight[j].seen << -off : 0);
    const uint32_t old = off >= 0 ? 0u : off > -32 ? (1u << -off) - 1u : ~0u;
    const uint32_t left = lo <= 0 ? 0u : lo < 32 ? (1u << lo) - 1u : ~0u;
    return valid[j] ? ((uint32_t)nodes | (old & ~left)) & pages : ~0u;
  };
  // a step's softmax and value products from its scores, and the scores of the next step
  auto attend = [&](Scores& sc, Scores& sn, const uint8_t* stg, const uint8_t* nxt, int step) __attribute__((always_inline)) {
    u32x4_t kf[4];
    load_keys(kf, nxt);
    bool ok[2];
    page_of(step, 0, ok[0]);
    page_of(step, 1, ok[1]);
    const int pg = it.pg0 + 2 * step, k0 = pg * PAGE;
    const bool second = pg + 1 < it.pg1;
    const bool edge = k0 + 2 * PAGE > it.len || (P.window > 0 && k0 < it.len + it.n - P.window) || !ok[0] || !ok[1] || !second;
    uint32_t vis[2];
    if (__builtin_expect(edge, 0)) {  // wave-uniform; the empty asm keeps it a branch
      asm volatile("");
      if ((!ok[0] || (!ok[1] && second)) && lane == 0) set_error(P.err, 1);
      const uint32_t pages = (ok[0] ? 0xFFFFu : 0u) | (ok[1] && second ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        vis[j] = visible(j, k0, pages);
        const uint32_t mine = vis[j] >> (4 * h);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc.t[j][e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? sc.t[j][e] : -INFINITY;
      }
    }
    u32x4_t pw[2][2];  // [column tile][page]: the weights, packed
    float sum[2];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sum[j] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sc.t[j][e], P.scale_log2, -m_sub[j]));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(sc.t[j][e + 1], P.scale_log2, -m_sub[j]));
          const uint32_t w = pack_bf16(p0, p1);
          pw[j][e >> 3][(e & 7) >> 1] = w;
          sum[j] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), sum[j], false);
        }
      }
    };
    __builtin_amdgcn_sched_barrier(0);
    scores(sn, kf);
    weights();
    // the next scores' eight products among the 96 vector instructions of the weights
#define TREE_MIX                                      \
  __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  \
  __builtin_amdgcn_sched_group_barrier(0x402, 12, 0);
    TREE_MIX TREE_MIX TREE_MIX TREE_MIX TREE_MIX TREE_MIX TREE_MIX TREE_MIX
#undef TREE_MIX
    // The maximum only has to keep the weights in range, so it is raised when a step's sum says that they are
    // not, and until a column has seen a key; the weights are then formed again.
    const bool raise = sum[0] > limit[0] || sum[1] > limit[1];
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {  // wave-uniform (kept a branch)
      asm volatile("");
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float mloc = sc.t[j][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mloc = vmax(mloc, sc.t[j][e]);
        const uint32_t u = __float_as_uint(mloc);
        auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        const float mstep = vmax(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * P.scale_log2;
        // a column's own lanes decide, so that its bits do not depend on the columns beside it
        const uint32_t o = sum[j] > limit[j];
        auto so = __builtin_amdgcn_permlane32_swap(o, o, false, false);
        const float m_new = (so[0] | so[1]) ? fmaxf(m_run[j], mstep) : m_run[j];
        const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[j] - m_new);
        l[j] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) acc[dt][j] *= alpha;
        m_run[j] = m_new;
        m_sub[j] = m_new == -INFINITY ? 0.f : m_new;  // masked scores give 2^-inf = 0
        limit[j] = m_new == -INFINITY ? -INFINITY : WEIGHT_LIMIT;
      }
      weights();
    }
    u32x4_t vf[2][2];  // [page][dim tile]
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int dt = 0; dt < 2; ++dt) {
        const uint8_t* v = stg + (2 + p) * PB + 1024 * dt + vbase;
        const u32x2_t a = *reinterpret_cast<const u32x2_t*>(v), c = *reinterpret_cast<const u32x2_t*>(v + 256);
        vf[p][dt] = __builtin_shufflevector(a, c, 0, 1, 2, 3);
      }
    if (__builtin_expect(edge, 0)) {
      asm volatile("");
      bool odd = false;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w = vf[p][dt][i];
            odd |= drop_nonfinite(w);
            vf[p][dt][i] = w;
          }
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {  // rare: values that are not finite, for the columns that see them
        for (int key = 0; key < 2 * PAGE; ++key) {
          const uint8_t* page = stg + (2 + (key >> 4)) * PB;
          const int slot = key & 15;
#pragma unroll
          for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int dim = 32 * dt + 8 * (e >> 2) + 4 * h + (e & 3);
              const uint32_t at = 2 * v_off(slot, dim);
              const uint16_t bits = *reinterpret_cast<const uint16_t*>(page + (at ^ (((at >> 9) & 1u) << 7)));
              const bool bad = (bits & 0x7F80u) == 0x7F80u;
#pragma unroll
              for (int j = 0; j < 2; ++j)
                acc[dt][j][e] += bad && (vis[j] >> key & 1) ? bf16_to_f32(bits) : 0.f;
            }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      l[j] += sum[j];
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
          acc[dt][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf[p][dt]),
                                                               __builtin_bit_cast(bf16x8_t, pw[j][p]), acc[dt][j], 0, 0, 0);
    }
  };

  // Step s sits in stage s % TRS. In step s its scores are there already; step s + TRS - 1 is requested into the
  // stage step s - 1 left, the scores of step s + 1 are formed, and before the barrier a wavefront waits for its
  // loads of step s + 2. The barrier hands the stages over: this wavefront's reads of the step's stage have
  // returned (lgkmcnt), its loads of step s + 2 have landed, and the empty asm keeps LDS accesses on their side.
  auto publish = [&]() __attribute__((always_inline)) {
    constexpr int N = LD * (TRS - 3);  // loads that may stay in flight
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (N >> 4 << 14));  // vmcnt(N) expcnt(7) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int s = 0; s < TRS - 1; ++s) {
    request(stage_of(s), s);
    __builtin_amdgcn_sched_barrier(0);
  }
  publish();
  Scores sc[2];
  if (busy) {
    u32x4_t kf[4];
    load_keys(kf, s0);
    scores(sc[0], kf);
  }
  auto one = [&](auto U_, int step) __attribute__((always_inline)) {
    constexpr int U = decltype(U_)::value;
    if (step < n_steps) {  // uniform
      request(stage_of((U + TRS - 1) % TRS), step + TRS - 1);
      if (busy) attend(sc[U % 2], sc[(U + 1) % 2], stage_of(U), stage_of((U + 1) % TRS), step);
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

  // this lane's dims 32 dt + 8 q + 4 h .. + 3 of each column: a partial row, or o with the sink
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t u = __float_as_uint(l[j]);
    auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    float l_tot = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (!valid[j]) continue;
    if (it.splits > 1) {
      const int64_t row = (int64_t)(it.row0 + node[j]) * P.hq + head[j];
      if (h == 0) *reinterpret_cast<float2*>(P.part_ml + 2 * row) = make_float2(m_run[j], l_tot);
#pragma unroll
      for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(P.part_acc + row * D + 32 * dt + 8 * q + 4 * h) =
              make_float4(acc[dt][j][4 * q], acc[dt][j][4 * q + 1], acc[dt][j][4 * q + 2], acc[dt][j][4 * q + 3]);
      continue;
    }
    float f = 1.0f;
    if (P.sinks) {
      const float sk = P.sinks[head[j]] * LOG2E, M = fmaxf(m_run[j], sk);
      f = m_run[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[j] - M);
      l_tot = l_tot * f + __builtin_amdgcn_exp2f(sk - M);
    }
    const float inv = l_tot == 0.f ? 0.f : f / l_tot;
    bf16* o = reinterpret_cast<bf16*>(P.o) + ((int64_t)(it.t0 + node[j]) * P.hq + head[j]) * D + 4 * h;
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store4(o + 32 * dt + 8 * q, make_float4(acc[dt][j][4 * q] * inv, acc[dt][j][4 * q + 1] * inv,
                                                acc[dt][j][4 * q + 2] * inv, acc[dt][j][4 * q + 3] * inv));
  }
}

template <int NC, int TRS>
static hipError_t tree_wide_impl(const TreeAttn& p, hipStream_t s) {
  const int cols = p.max_nodes * (p.hq / p.hkv), tiles = (cols + 64 * NC - 1) / (64 * NC);
  const int64_t blocks = (int64_t)p.n_items * p.hkv * tiles;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL((tree_attn_wide_kernel<NC, TRS>), dim3((unsigned)blocks), dim3(64 * NC), 0, s, p, tiles);
  return hipGetLastError();
}

hipError_t launch_tree_attn(int dtype, int head_dim, const TreeAttn& p, hipStream_t s) {
  if (p.n_items == 0) return hipSuccess;
  // bf16 with head dim 64 takes the wide products, whose pages go to LDS by 16-byte direct loads: 16-byte
  // aligned pools only. As many wavefronts as the largest tree has columns share a page.
  if (dtype == 1 && head_dim == 64 && ((uintptr_t)p.k_pool | (uintptr_t)p.v_pool) % 16 == 0) {
    const int cols = p.max_nodes * (p.hq / p.hkv);
    if (cols <= 64) return tree_wide_impl<1, 4>(p, s);
    if (cols <= 128) return tree_wide_impl<2, 6>(p, s);
    if (cols <= 256) return tree_wide_impl<4, 6>(p, s);
    return tree_wide_impl<8, 6>(p, s);
  }
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
