// What the two kernels of attention over the paged cache share (kv_attention.cu, kv_attention_wide.cu): the walk
// over a CTA's runs of tiles, what travels beside a tile, where a tile's rows lie.
#pragma once

#include "kv_internal.cuh"

namespace lif {

struct AttendArgs {
  const void *q, *pages;       // pages: this layer's
  void* out;
  float scale_log2;            // scale * log2(e): weights are powers of two
  int layer;
};

// What a stage of the ring holds.
struct __align__(16) StageInfo {
  int b, tokens, news, k0;     // place, its tokens, its new ones, first key
  int head, row0, flags;       // key-value head, first row of the row block
  int run;
};
// first tile of a piece, of the head; last tile of the head, of a piece, of the CTA; keys that not every row sees
enum { kOpens = 1, kStarts = 2, kEnds = 4, kCloses = 8, kLast = 16, kEdge = 32 };

// 2^x; results below 2^-126 are 0 (a weight that small is none in 16 bits)
__device__ __forceinline__ float power(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Weights are 2^(score - reference).  The reference need not be the row's maximum, only near enough that no weight is
// too large; it is brought up to date, and what was summed scaled down, when a score lies more than kSlack above the
// one that set it.  That one has weight 2^kLift, so nothing gets smaller than with the maximum.  The lift is for fp16,
// which holds 2^-24 .. 65504: weights go up to 2^(kLift + kSlack) = 2^15, and what is far below the largest one
// counts down to 2^-32 of it, where without the lift all keys below 2^-25 would be lost: a quarter (narrow kernel) to
// nearly all (wide) of the output where one key of no value holds the weight and 131001 others lie there.  It costs nothing:
// it stands in the reference.
// What is compared is the exponent of the row's largest weight, formed as every weight's is (one rounding; no weight
// has a larger one), and a new reference is rounded up: then no exponent passes kLift + kSlack however coarse fp32 is
// at that score.  (A product rounded on its own and a rounded reference + slack let weights of 2^16 through at 2^27.)
constexpr float kSlack = 8.f;
template <typename T>
__device__ __forceinline__ bool too_far(float top, float scale, float reference) {   // (false where both are -inf)
  return fmaf(top, scale, -reference) > kSlack + Num<T>::kLift;
}
template <typename T>
__device__ __forceinline__ float new_reference(float top, float scale) { return __fmaf_ru(top, scale, -Num<T>::kLift); }

// a box of the pool at {column, row in the page, operand and head, page, layer}
__device__ __forceinline__ void tensor_g2s(uint32_t to, const CUtensorMap* map, int x, int row, int head, int page,
                                           int layer, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5,%6}], [%7];"
      ::"r"(to), "l"(map), "r"(x), "r"(row), "r"(head), "r"(page), "r"(layer), "r"(smem_u32(bar))
      : "memory");
}

// Byte where 16-byte piece c of row r lies in a tile of 64 rows of D elements: 64 columns after 64, the rest
// behind them; within 128 (64) bytes of a row the pieces are permuted by the row as the tensor map's swizzle
// does it.  Rows of 80 elements lie as they are: only rows r and r + 4 meet in a bank, and one copy
// a page and operand in place of two, the second 32 bytes wide, takes 15.9 us where two took 16.5 (8 sequences, 32
// heads, five tokens).
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  if (D == 80) return r * 160 + c * 16;
  if (c < D / 64 * 8) return (c / 8) * 8192 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
  return D / 64 * 8192 + r * 64 + (((c & 3) ^ (r >> 1 & 3)) << 4);
}
// the same for piece c0 + b, c0 even and known, b 0 or 1
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c0, int b) {
  if (D == 80) return r * 160 + b * 16 + c0 * 16;
  if (c0 < D / 64 * 8) return (c0 / 8) * 8192 + r * 128 + (((c0 & 7) ^ (b ^ (r & 7))) << 4);
  return D / 64 * 8192 + r * 64 + (((c0 & 3) ^ (b ^ (r >> 1 & 3))) << 4);
}

// A place in the step's work.
struct Cursor {
  int b, tokens, news, tiles, blocks, head, block, tile, first_tile;
  __device__ __forceinline__ void enter(const KvView& V, int place, int n_tokens, int n_new) {
    b = place;
    tokens = n_tokens;
    news = n_new;
    tiles = kv_tiles(n_tokens, n_new, V.window);
    blocks = kv_row_blocks(n_new, V.group, V.rows_per_block);
    first_tile = kv_first_key(n_tokens, n_new, V.window) / kKvTile;
  }
  __device__ __forceinline__ void step(const KvView& V) {
    if (++tile < tiles) return;
    tile = 0;
    if (++block < blocks) return;
    block = 0;
    if (++head < V.n_kv_heads) return;
    head = 0;
    for (int p = b + 1; p < V.max_seqs; ++p) {
      const int4 s = V.seq_plan[p];
      if (s.w > 0) {
        enter(V, p, s.y, s.z);
        return;
      }
    }
  }
};

// A CTA's way through its runs, tile by tile: its first run, then further ones while there are any (kv_plan).
// The 32 lanes of one warp walk together.
struct Walk {
  Cursor at;
  int total, share, first_tiles, more_tiles, more, n_more;
  int run, next, g, end;
  int held_b, held_from, held;                       // 32 page ids of a place, one a lane
  bool opens_run, opens, ends_run, last;
  int k0, j0, n_pages;                               // first key, its page in the table, pages with keys of this tile

  // who: the CTA's number (or that of a half of one); plan: its first run's entry of run_plan; step: counts[KV_TILES ..]
  __device__ __forceinline__ Walk(const KvView& V, int who, int4 plan, int4 step) {
    total = step.x;
    share = step.z;
    first_tiles = step.w;
    const int4 others = *reinterpret_cast<const int4*>(V.counts + KV_MORE_TILES);
    more_tiles = others.x;
    more = others.y;
    n_more = others.z;
    run = who * (1 + more);
    next = 0;
    g = who * share;
    end = min(total, g + first_tiles);
    held_b = held_from = -1;
    held = 0;
    opens_run = true;
    last = false;
    seek(V, plan);
  }
  __device__ __forceinline__ void seek(const KvView& V, const int4& p) {
    at.enter(V, p.x, p.z, p.w);
    const int in = g - p.y, item = in / at.tiles;
    at.tile = in - item * at.tiles;
    at.head = item / at.blocks;
    at.block = item - at.head * at.blocks;
  }
  __device__ __forceinline__ void begin(const KvView& V, int lane) {
    k0 = (at.first_tile + at.tile) * kKvTile;
    j0 = k0 >> V.page_shift;
    const int pages = kv_pages_of(at.tokens, V.page_shift);
    n_pages = min(pages - j0, max(1, kKvTile >> V.page_shift));
    if (at.b != held_b || (j0 & ~31) != held_from) {
      held_b = at.b;
      held_from = j0 & ~31;
      held = held_from + lane < pages ? V.table[(size_t)at.b * V.max_pages + held_from + lane] : 0;
    }
    opens = opens_run || at.tile == 0;
    if (opens_run) {                                 // the run after this one; asked for long before it is needed
      if (n_more && lane == 0) next = atomicAdd(V.counts + KV_TAKEN, 1);
      opens_run = false;
    }
    ends_run = g + 1 == end;
    if (ends_run) {
      next = __shfl_sync(~0u, next, 0);
      last = next >= n_more;
    }
  }
  __device__ __forceinline__ StageInfo info(const KvView& V) const {
    const bool ends = at.tile + 1 == at.tiles;
    StageInfo n;
    n.b = at.b;
    n.tokens = at.tokens;
    n.news = at.news;
    n.k0 = k0;
    n.head = at.head;
    n.row0 = at.block * V.rows_per_block;
    n.flags = (opens ? kOpens : 0) | (at.tile == 0 ? kStarts : 0) | (ends ? kEnds : 0) | (ends || ends_run ? kCloses : 0) |
              (last ? kLast : 0) |
              (k0 + kKvTile > at.tokens - at.news + 1 || (V.window > 0 && k0 <= at.tokens - 1 - V.window) ? kEdge : 0);
    n.run = run;
    return n;
  }
  __device__ __forceinline__ void advance(const KvView& V) {
    if (!ends_run) {
      ++g;
      at.step(V);
    } else if (!last) {
      const int c = next / more, j = next - c * more;
      run = c * (1 + more) + 1 + j;
      g = c * share + first_tiles + j * more_tiles;
      end = min(min(total, c * share + share), g + more_tiles);
      opens_run = true;
      seek(V, V.run_plan[V.ctas + next]);
    }
  }
};

// Does a tile hold keys that some rows see and others do not, or that none sees?  Keys [some, all) and [few, end) are
// seen by some, those before and behind by none; of the keys [first, first + n):
struct Edge {
  int some, all, few;
  __device__ __forceinline__ Edge(const KvView& V, const StageInfo& at) {
    some = kv_first_key(at.tokens, at.news, V.window);
    all = V.window > 0 ? at.tokens - V.window : 0;
    few = at.tokens - at.news + 1;
  }
  __device__ __forceinline__ bool none(const StageInfo& at, int key) const { return key < some || key >= at.tokens; }
  __device__ __forceinline__ bool clear(const StageInfo& at, int first, int n) const {
    return first < some || first + n > at.tokens;
  }
  __device__ __forceinline__ bool differ(const StageInfo& at, int first, int n) const {
    return at.news > 1 && (first < all || first + n > few);
  }
};
template <typename T>
__device__ __forceinline__ bool any_not_finite(const uint4& v) {
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t y = (&v.x)[e], lo = Num<T>::kExponent & 0xffffu, hi = Num<T>::kExponent & 0xffff0000u;
    odd = odd || (y & lo) == lo || (y & hi) == hi;
  }
  return odd;
}
// Row r's place in queries and output: token t = (row0 + r) / group, head (row0 + r) % group of the key-value head's.
__device__ __forceinline__ int64_t row_offset(const KvView& V, const StageInfo& at, int r) {
  const int t = (at.row0 + r) / V.group, h = at.row0 + r - t * V.group;
  return (((int64_t)at.b * V.max_new + t) * V.n_heads + at.head * V.group + h) * V.head_dim;
}

// kv_attention_wide.cu
inline bool kv_is_wide(const lif_kv_desc& d) { return (d.head_dim == 64 || d.head_dim == 128) && kv_row_tiles(d) > 1; }
cudaError_t kv_wide_configure(const lif_kv* kv, int* ctas_per_sm);
cudaError_t launch_kv_attention_wide(const lif_kv* kv, const AttendArgs& a, cudaStream_t st);

}  // namespace lif
