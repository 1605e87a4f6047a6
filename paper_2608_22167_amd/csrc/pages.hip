// Moves inside the paged cache: an accepted path onto consecutive slots, and
// whole pages into other pages, for every layer that shares the page ids in one
// launch.
#include "device.h"
#include "kernels_tree.h"

namespace mcpu {

// ---------------------------------------------------------------------------
// commit: slot len + path[i] -> slot len + i, i < n_path
// ---------------------------------------------------------------------------

// A workgroup per (sequence, pool, KV head), four wavefronts. A path ascends and
// path[i] >= i, so its first nodes are often in place: only rows from the first
// i with path[i] != i move. Slots are both read and written by one path (slot i
// may be the source of an earlier row), so all rows are read, then a barrier, then
// all are written; other workgroups touch other heads or pages. A path that does
// not ascend inside its tree raises bit 64 and moves nothing, a missing page bit
// 1 and drops its row. Bound by latency: the table and the path, then one round of
// loads and one of stores.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_commit_kernel(TreeCommit P) {
  constexpr int N = TREE_MAX_NODES;
  __shared__ int64_t from[N], to[N];  // element offset of the page's head block, or -1
  __shared__ int slot_from[N], slot_to[N];
  const int b = blockIdx.x, pool = blockIdx.y, g = blockIdx.z, tid = threadIdx.x, lane = lane_id();
  const int t0 = P.cu_q[b], n = P.cu_q[b + 1] - t0, len = P.seq_lens[b], m = P.n_path[b];
  if (n < 0 || n > N || t0 < 0 || t0 + n > P.n_tokens || len < 0 || m < 0 || m > n) {
    if (tid == 0) set_error(P.err, 8);
    return;
  }
  // every wavefront checks the path for itself (lane i: row i)
  const int node = lane < m ? P.path[t0 + lane] : 0;
  const int before = __shfl_up(node, 1, 64);
  const bool wrong = lane < m && (node < lane || node >= n || (lane > 0 && node <= before));
  if (__ballot(wrong) != 0) {
    if (tid == 0) set_error(P.err, 64);
    return;
  }
  const uint64_t moved = __ballot(lane < m && node != lane);
  if (moved == 0) return;
  const int first = (int)__builtin_ctzll(moved), rows = m - first;
  if (tid < N && lane >= first && lane < m) {
    const int s = len + node, d = len + lane;
    const int32_t* row = P.page_table + (int64_t)b * P.max_pages;
    const int ps = s / PAGE < P.max_pages ? row[s / PAGE] : -1, pd = d / PAGE < P.max_pages ? row[d / PAGE] : -1;
    const bool ok = ps >= 0 && ps < P.n_pages && pd >= 0 && pd < P.n_pages;
    if (!ok) set_error(P.err, 1);
    from[lane - first] = ok ? ((int64_t)ps * P.hkv + g) * PAGE * D : -1;
    to[lane - first] = ok ? ((int64_t)pd * P.hkv + g) * PAGE * D : -1;
    slot_from[lane - first] = s % PAGE;
    slot_to[lane - first] = d % PAGE;
  }
  __syncthreads();
  T* kp = reinterpret_cast<T*>(P.pools.k[pool]);
  T* vp = reinterpret_cast<T*>(P.pools.v[pool]);
  constexpr int U = N * D / 256;  // elements per thread of K, and of V
  T k[U], v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = tid + 256 * u, r = e / D, i = e % D;
    if (r < rows && from[r] >= 0) {
      k[u] = kp[from[r] + k_off(slot_from[r], i)];
      v[u] = vp[from[r] + v_off(slot_from[r], i)];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = tid + 256 * u, r = e / D, i = e % D;
    if (r < rows && from[r] >= 0) {
      kp[to[r] + k_off(slot_to[r], i)] = k[u];
      vp[to[r] + v_off(slot_to[r], i)] = v[u];
    }
  }
}

hipError_t launch_tree_commit(int dtype, int head_dim, const TreeCommit& p, hipStream_t s) {
  if (p.batch == 0) return hipSuccess;
  const dim3 grid(p.batch, p.n_pools, p.hkv), block(256);
  if (dtype == 0) {
    if (head_dim == 32) hipLaunchKernelGGL((tree_commit_kernel<float, 32>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_commit_kernel<float, 64>), grid, block, 0, s, p);
  } else {
    if (head_dim == 32) hipLaunchKernelGGL((tree_commit_kernel<bf16, 32>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_commit_kernel<bf16, 64>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// copy: page src[i] -> page dst[i]
// ---------------------------------------------------------------------------

// A workgroup per (pair, pool, K or V). Bound by HBM: a page is read and written
// once.
template <typename V>
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopy P) {
  const int i = blockIdx.x, pool = blockIdx.y;
  const int s = P.src[i], d = P.dst[i];
  if (s < 0 || s >= P.n_pages || d < 0 || d >= P.n_pages) {
    if (threadIdx.x == 0) set_error(P.err, 1);
    return;
  }
  char* base = reinterpret_cast<char*>(blockIdx.z ? P.pools.v[pool] : P.pools.k[pool]);
  const V* from = reinterpret_cast<const V*>(base + s * P.page_bytes);
  V* to = reinterpret_cast<V*>(base + d * P.page_bytes);
  for (int c = threadIdx.x; c < (int)(P.page_bytes / (int64_t)sizeof(V)); c += 256) to[c] = from[c];
}

hipError_t launch_pages_copy(const PagesCopy& p, hipStream_t s) {
  if (p.n == 0) return hipSuccess;
  const dim3 grid(p.n, p.n_pools, 2), block(256);
  uintptr_t all = (uintptr_t)p.page_bytes;
  for (int i = 0; i < p.n_pools; ++i) all |= (uintptr_t)p.pools.k[i] | (uintptr_t)p.pools.v[i];
  if (all % 16 == 0) hipLaunchKernelGGL(pages_copy_kernel<uint4>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(pages_copy_kernel<uint16_t>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace mcpu
