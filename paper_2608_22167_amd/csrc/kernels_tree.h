// Internal launch interface of the drafted-token-tree and cache-page kernels
// (tree.hip, pages.hip). Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mcpu {

constexpr int TREE_MAX_NODES = 64;  // a node's ancestors are the bits of one 64-bit word

// One split of a tree's visible pages: n nodes (rows t0 ..) of sequence b (-1: no
// split) behind len committed tokens, logical pages pg0 .. pg1 - 1. Its partial rows
// (node i of part_ml / part_acc at row0 + i) exist where the tree has more than one
// split; a tree's only split writes o itself.
struct TreeItem {
  int32_t b, t0, n, len, pg0, pg1, row0, splits;
};
constexpr int TREE_SCAN = 256;  // up to this many sequences the items are found without a plan launch

struct TreeArgs {
  const int32_t* seq_lens;  // [batch]
  const int32_t* cu_q;      // [batch + 1]
  const int32_t* parents;   // [n_tokens]
  int batch, n_tokens, max_pages, window;
  int max_nodes;            // of a tree, as the host counted them
  int pps;                  // pages per split
  int n_items, n_rows;      // splits and partial rows as the host counted them, checked on the device; without
                            // partial rows item i is tree i (n_items = batch)
  const TreeItem* item;     // [n_items] from the plan kernel, or nullptr
  int4* tok;                // [n_tokens] where n_rows > 0: first partial row, rows per split, splits (0: no such tree)
  int32_t* err;
};
hipError_t launch_tree_plan(const TreeArgs& p, TreeItem* out, hipStream_t s);

// How a step's columns (node and query head pairs of one KV head) are dealt out:
// `cols` of them to each workgroup (each wavefront for TREE_ANY), of which `per_cu`
// are at work on a compute unit at a time.
enum TreeKind { TREE_ANY, TREE_NARROW, TREE_NARROW_STREAM, TREE_WIDE1, TREE_WIDE2, TREE_WIDE4 };
struct TreeForm {
  int kind, cols, per_cu;
};
TreeForm tree_attn_form(int dtype, int head_dim, const void* k_pool, const void* v_pool, int cols, bool few, bool one_each);

struct TreeAttn : TreeArgs {
  const void* q;  // [n_tokens][Hq][D]
  const void* k_pool;
  const void* v_pool;
  const int32_t* page_table;
  int n_pages, hq, hkv;
  TreeForm form;
  float scale_log2;    // log2(e) / sqrt(D)
  const float* sinks;  // [Hq] or nullptr
  float* part_ml;      // [n_rows][Hq][2] running max (log2 units) and sum
  float* part_acc;     // [n_rows][Hq][D]
  void* o;             // [n_tokens][Hq * D]
};
hipError_t launch_tree_attn(int dtype, int head_dim, const TreeAttn& p, hipStream_t s);

// rope[t] = len + depth of each node: the position its q and k are rotated at
hipError_t launch_tree_positions(const TreeArgs& p, int32_t* rope, hipStream_t s);

struct TreeCombine {
  const float* part_ml;
  const float* part_acc;
  const int4* tok;
  const float* sinks;
  int n_tokens, n_rows, hq;
  int max_splits;  // of a tree
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
