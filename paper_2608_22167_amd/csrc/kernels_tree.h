// Internal launch interface of the drafted-token-tree and cache-page kernels
// (tree.hip, pages.hip). Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mcpu {

constexpr int TREE_MAX_NODES = 64;  // a node's ancestors are the bits of one 64-bit word

// Node i of its tree: bit a of `seen` is set if node a is an ancestor of i (or
// i itself) inside i's window; depth = ancestors without i.
struct TreeNode {
  uint64_t seen;
  int32_t depth, pad;
};

// One split of a tree's visible pages: n nodes (rows t0 ..) of sequence b behind
// len committed tokens, logical pages pg0 .. pg1 - 1. Its partial rows (node i of
// part_ml / part_acc at row0 + i) exist where the tree has more than one split
// (splits > 1); a tree's only split writes o itself.
struct TreeItem {
  int32_t b, t0, n, len, pg0, pg1, row0, splits;
};

struct TreePlan {
  const int32_t* seq_lens;  // [batch]
  const int32_t* cu_q;      // [batch + 1]
  const int32_t* parents;   // [n_tokens]
  int batch, n_tokens, max_pages, window, pps;
  int n_items, n_rows;      // what the host planned; checked on the device
  TreeNode* node;           // [n_tokens] out
  TreeItem* item;           // [n_items] out
  int32_t* tok_seq;         // [n_tokens] out
  int2* seq_split;          // [batch] out: first partial row, number of splits
  int32_t* err;
};
hipError_t launch_tree_plan(const TreePlan& p, hipStream_t s);

struct TreeAttn {
  const void* q;  // [n_tokens][Hq][D]
  const void* k_pool;
  const void* v_pool;
  const int32_t* page_table;
  int max_pages, n_pages;
  const TreeNode* node;
  const TreeItem* item;
  int batch, n_tokens, n_items, n_rows, max_nodes, hq, hkv, window;
  float scale_log2;    // log2(e) / sqrt(D)
  const float* sinks;  // [Hq] or nullptr
  float* part_ml;      // [n_rows][Hq][2] running max (log2 units) and sum
  float* part_acc;     // [n_rows][Hq][D]
  void* o;             // [n_tokens][Hq * D]
  int32_t* err;
};
hipError_t launch_tree_attn(int dtype, int head_dim, const TreeAttn& p, hipStream_t s);

struct TreeCombine {
  const float* part_ml;
  const float* part_acc;
  const int32_t* cu_q;
  const int32_t* tok_seq;
  const int2* seq_split;
  const float* sinks;
  int batch, n_tokens, n_rows, hq;
  void* o;
};
hipError_t launch_tree_combine(int dtype, int head_dim, const TreeCombine& p, hipStream_t s);

struct TreeAccept {
  const int32_t* cu_q;
  const int32_t* parents;
  const int32_t* draft;
  const int32_t* sampled;
  int batch, n_tokens;
  int32_t* path;    // [n_tokens]
  int32_t* n_path;  // [batch]
  int32_t* next;    // [batch]
  int32_t* err;
};
hipError_t launch_tree_accept(const TreeAccept& p, hipStream_t s);

// The K and V pools of up to MAX_POOLS layers that share one page-id space.
constexpr int MAX_POOLS = 64;
struct PoolSet {
  void* k[MAX_POOLS];
  void* v[MAX_POOLS];
};

struct TreeCommit {
  PoolSet pools;
  int n_pools, n_pages, hkv;
  const int32_t* page_table;
  int max_pages;
  const int32_t* seq_lens;
  const int32_t* cu_q;
  const int32_t* path;    // [n_tokens]
  const int32_t* n_path;  // [batch]
  int batch, n_tokens;
  int32_t* err;
};
hipError_t launch_tree_commit(int dtype, int head_dim, const TreeCommit& p, hipStream_t s);

struct PagesCopy {
  PoolSet pools;
  int n_pools, n_pages, n;
  const int32_t* src;  // [n]
  const int32_t* dst;  // [n]
  int64_t page_bytes;  // of K (or V) of one page
  int32_t* err;
};
hipError_t launch_pages_copy(const PagesCopy& p, hipStream_t s);

}  // namespace mcpu
