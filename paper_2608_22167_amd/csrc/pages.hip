// Moves inside the paged cache: an accepted path onto consecutive slots, and
// whole pages into other pages, for every layer that shares the page ids in one
// launch.
#include "device.h"
#include "kernels_tree.h"

namespace mcpu {

// ---------------------------------------------------------------------------
// commit: slot len + path[i] -> slot len + i, i < n_path
// ---------------------------------------------------------------------------

// A workgroup per (sequence, pool, KV head). A path ascends and path[i] >= i, so its
// first nodes are often in place, and only rows from the first i with path[i] != i on
// move, 16 at a time: all read, a barrier, all written. A row is never written before
// it is read: slot i is the source of rows up to i alone, and rows behind the 16 have
// sources behind them. A path that does not ascend inside its tree raises bit 64 and
// moves nothing, a missing page bit 1 and drops its row.
//
// Bound by latency: three rounds of loads one after the other (row offsets; path and
// pages; data). 48 sequences of up to 16 nodes, twelve layers: 8.8 us, and 4.4 for
// three in one layer. One wavefront per head instead of four took 15 us, 16-byte
// pieces of K instead of single elements, a lane of a store each on a line of its own,
// 16.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_commit_kernel(TreeCommit P) {
  constexpr int R = 16, U = R * D / 256;                      // rows per turn, elements of K and of V per thread
  constexpr int NP = (TREE_MAX_NODES + PAGE - 2) / PAGE + 1;  // pages that a tree's slots touch
  const int b = blockIdx.x, pool = blockIdx.y, g = blockIdx.z, tid = threadIdx.x, lane = lane_id();
  const int t0 = P.cu_q[b], n = P.cu_q[b + 1] - t0, len = P.seq_lens[b], m = P.n_path[b];
  if (n < 0 || n > TREE_MAX_NODES || t0 < 0 || t0 > P.n_tokens - n || len < 0 || len > INT32_MAX - TREE_MAX_NODES ||
      m < 0 || m > n) {
    if (tid == 0) set_error(P.err, 8);
    return;
  }
  // every wavefront for itself, lane i: the tree's page i, and row i
  const int pg = len / PAGE + lane;
  int id = lane < NP && pg < P.max_pages ? P.page_table[(int64_t)b * P.max_pages + pg] : -1;
  id = id < P.n_pages ? id : -1;
  const int node = lane < m ? P.path[t0 + lane] : 0;
  const int before = __shfl_up(node, 1, 64);
  if (__ballot(lane < m && (node < lane || node >= n || (lane > 0 && node <= before))) != 0) {
    if (tid == 0) set_error(P.err, 64);
    return;
  }
  const uint64_t moved = __ballot(lane < m && node != lane);
  if (moved == 0) return;
  // where row i's elements lie on either side: page * 16 + slot, or NONE where a page is missing
  constexpr uint32_t NONE = ~0u;  // beyond any pool that fits the GPU
  const int src = len % PAGE + node, dst = len % PAGE + min(lane, TREE_MAX_NODES - 1);
  const int ps = __shfl(id, src / PAGE, 64), pd = __shfl(id, dst / PAGE, 64);
  const bool there = ps >= 0 && pd >= 0;
  if (tid < m && node != lane && !there) set_error(P.err, 1);
  const uint32_t from = there ? (uint32_t)ps * PAGE + src % PAGE : NONE, to = there ? (uint32_t)pd * PAGE + dst % PAGE : NONE;
  T* kp = reinterpret_cast<T*>(P.pools.k[pool]);
  T* vp = reinterpret_cast<T*>(P.pools.v[pool]);
  auto block = [&](uint32_t place) __attribute__((always_inline)) { return ((int64_t)(place / PAGE) * P.hkv + g) * PAGE * D; };
  for (int i0 = (int)__builtin_ctzll(moved); i0 < m; i0 += R) {
    T k[U], v[U];
    // loads without a condition, all of a turn's in flight together: rows past the path read its last one, missing
    // ones the pool's first slot
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = tid + 256 * u, i = e % D;
      uint32_t x = __shfl(from, min(i0 + e / D, m - 1), 64);
      x = x == NONE ? 0 : x;
      k[u] = kp[block(x) + k_off(x % PAGE, i)];
      v[u] = vp[block(x) + v_off(x % PAGE, i)];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = tid + 256 * u, i = e % D, row = i0 + e / D;
      const uint32_t x = __shfl(to, min(row, m - 1), 64);
      if (row < m && x != NONE) {
        kp[block(x) + k_off(x % PAGE, i)] = k[u];
        vp[block(x) + v_off(x % PAGE, i)] = v[u];
      }
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
// once, 1500 pages of 8 KV heads in two layers in 31.9 us (6.2 TB/s read and
// written; a large copy 4.9, this one fits the last-level cache).
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

// do all pools of a set start on 16-byte boundaries?
static bool aligned16(const PoolSet& p, int n) {
  uintptr_t all = 0;
  for (int i = 0; i < n; ++i) all |= (uintptr_t)p.k[i] | (uintptr_t)p.v[i];
  return all % 16 == 0;
}

hipError_t launch_pages_copy(const PagesCopy& p, hipStream_t s) {
  if (p.n == 0) return hipSuccess;
  const dim3 grid(p.n, p.n_pools, 2), block(256);
  if (aligned16(p.pools, p.n_pools)) hipLaunchKernelGGL(pages_copy_kernel<uint4>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(pages_copy_kernel<uint16_t>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace mcpu
