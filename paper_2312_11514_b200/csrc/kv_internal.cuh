// Internal declarations of the paged key-value cache (lif_kv.h): kv.cu (calls and tables),
// kv_append.cu, kv_attention.cu.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "lif_internal.cuh"
#include "lif_kv.h"

namespace lif {

constexpr int kKvTile = 64;          // keys per tile of the attention kernel
constexpr int kKvMaxCtas = 320;      // its CTAs, at most
constexpr int kKvMaxRuns = 2048;     // and their runs of tiles
constexpr int kKvPlanThreads = 1024; // threads of the kernels that change the tables
constexpr int kKvCluster = 8;        // CTAs of those that work on whole tables

// Private entries of the counts block.
enum {
  KV_FREE_FROM = 16,      // no free page has a lower id
  // the step's attention (kv_plan); two 16-byte loads
  KV_TILES = 20,          // tiles in all,
  KV_SHARES = 21,         // shares that they are cut into, one a CTA,
  KV_SHARE = 22,          // tiles of a share,
  KV_FIRST_TILES = 23,    // of them the CTA's first run,
  KV_MORE_TILES = 24,     // a further run,
  KV_MORE = 25,           // further runs of a share
  KV_MORE_IN_ALL = 26,    // and of all (the last share may have fewer),
  KV_JOINS = 27,          // entries of `joins`
  KV_TAKEN = 28           // further runs taken so far; 0 between calls
};

// Everything the kernels need of a cache, by value.
struct KvView {
  int32_t *counts, *lens, *n_new, *table, *refs;
  int32_t *table_tmp;      // [max_seqs][max_pages]
  int32_t *page_tmp;       // [n_pages] scratch per page
  int32_t *list_a, *list_b;  // [n_pages] lists of page ids; copies: source, destination ...
  int32_t *copy_tokens;    // [n_pages] ... and rows
  int4 *seq_plan;          // [max_seqs] {first tile, tokens, new tokens, tiles per row block}
  int4 *run_plan;          // [CTAs] of their first runs, [max_runs] of the others:
                           // {place, its first tile, tokens, new tokens} at the run's first tile
  int4 *joins;             // [max_runs] {first run, last run << 16; place; head << 16, row block; new tokens}
  const uint64_t* turns;   // [rope_dims/2] 2^64ths of a turn per position
  float* partials;         // [2 * max_runs][slot_rows] {[head_dim], reference, sum, -, -}
  int max_seqs, max_pages, n_pages, max_new, page_shift, window;
  int n_heads, n_kv_heads, group, head_dim, rows_per_block, ctas;
  int max_runs, slot_rows, slot_floats;
};

struct KvWorkspace {
  size_t counts, lens, n_new, table, table_tmp, refs, page_tmp, list_a, list_b, copy_tokens,
      seq_plan, run_plan, joins, turns, partials, total;
};

// The pool for tensor copies: boxes of 64 columns, and of those that head_dim % 64 leaves.
struct KvMaps {
  CUtensorMap wide, rest;
};

}  // namespace lif

struct lif_kv {
  lif_kv_desc desc;
  lif::KvView v;
  lif::KvMaps maps;
  int device, n_sm;
  int row_tiles;            // 16-row tiles per row block of the attention kernel
  float scale;
};

namespace lif {

// elements of one page of one layer
inline size_t kv_page_elems(const lif_kv_desc& d) {
  return (size_t)2 * d.n_kv_heads * d.page_tokens * d.head_dim;
}
int kv_row_tiles(const lif_kv_desc& d);
// rows of a row block that can be there
inline int kv_slot_rows(const lif_kv_desc& d) {
  const int rows = d.n_heads / d.n_kv_heads * d.max_new, block = 16 * kv_row_tiles(d);
  return rows < block ? rows : block;
}
// Runs of the attention kernel's work at most: where a block has few rows (and what its pieces leave
// behind is small), further ones beside a CTA's first.
inline int kv_max_runs(const lif_kv_desc& d) { return kv_slot_rows(d) <= 32 ? kKvMaxRuns : kKvMaxCtas; }
// Tensor maps, and CTAs per SM of the attention kernel for this cache
bool kv_attention_configure(lif_kv* kv, int* ctas_per_sm);
cudaError_t launch_kv_append(const lif_kv* kv, int layer, const lif_kv_rows& q, const lif_kv_rows& k,
                             const lif_kv_rows& v, const lif_kv_norms& norms, void* q_out, cudaStream_t st);
cudaError_t launch_kv_attention(const lif_kv* kv, int layer, const void* q, void* out, cudaStream_t st);

#ifdef __CUDACC__
__device__ __forceinline__ int kv_pages_of(int tokens, int shift) {
  return (int)(((unsigned)tokens + (1u << shift) - 1) >> shift);
}
// First key that any of the sequence's new tokens sees, and the tiles from there on.
__device__ __forceinline__ int kv_first_key(int tokens, int n_new, int window) {
  const int first = tokens - n_new + 1 - window;
  return window > 0 && first > 0 ? first : 0;
}
__device__ __forceinline__ int kv_tiles(int tokens, int n_new, int window) {
  return n_new > 0 ? (tokens + kKvTile - 1) / kKvTile - kv_first_key(tokens, n_new, window) / kKvTile : 0;
}
__device__ __forceinline__ int kv_row_blocks(int n_new, int group, int rows_per_block) {
  return (n_new * group + rows_per_block - 1) / rows_per_block;
}

// The two 16-bit types.
template <typename T> struct Num;
template <> struct Num<__half> {
  static __device__ __forceinline__ float2 to2(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
  static __device__ __forceinline__ uint32_t from2(float a, float b) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
  static constexpr uint32_t kExponent = 0x7c007c00u;   // all ones: infinite or NaN
  static constexpr float kLift = 7.f;                  // of a softmax's weights (kv_attention.cuh)
};
template <> struct Num<__nv_bfloat16> {
  static __device__ __forceinline__ float2 to2(uint32_t v) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&v)); }
  static __device__ __forceinline__ uint32_t from2(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
  static constexpr uint32_t kExponent = 0x7f807f80u;
  static constexpr float kLift = 0.f;
};
#endif

}  // namespace lif
