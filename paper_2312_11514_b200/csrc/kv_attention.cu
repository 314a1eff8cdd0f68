// Attention of a step's new tokens over the paged key-value cache.
//
//   out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale <q_row, k_j> - max_j)
//
// Rows: the new tokens' query heads that share a key-value head, `group` x tokens of them (1 .. 16
// mostly), in blocks of 16 x WR.  Every key and value is read once per row block; bound: HBM, until
// rows x heads make the tensor cores or the exponentials one (a single key-value head under many query heads).
//
// Split.  The step's work is numbered in tiles of 64 keys (kv_plan) and every CTA takes an equal run
// of them, across heads and sequences, so that one long sequence, many short ones and anything ragged
// between fill the chip alike.  A head that a run's end cuts is finished from the pieces' {max, sum,
// unnormalised output}, in the pieces' order, by the CTA that writes the last of them (a ticket per cut
// head); a second launch for it cost 3 us of device and 2 us of host time more.
//
// Loads.  One warp feeds the others: it walks the run, reads 32 page ids at a time and moves keys and
// values into a ring of stages with tensor copies (TMA), a copy per page, 64 columns and operand, which
// store a row's 16-byte pieces in the permuted order that makes ldmatrix free of bank conflicts.  What a
// stage holds (place, head, first key ...) travels beside it, so the other warps divide nothing.
// Tokens past the end lie in the same page and are copied too; the values among them are cleared in
// shared memory before use (whatever they hold, 0 times it is not 0), the scores replaced by -inf.
//
// Products.  Of 64 keys each of WK warps takes 64 / WK, of the rows each of WR warps 16, and keeps a
// running maximum, sum and output of its own (mma m16n8k16): between two tiles no warp waits for another,
// and the weights stay in registers from the first product to the second.  The WK warps of a row
// are summed when the head ends.
//
// Precision.  Scores, maxima, sums and outputs are fp32.  Weights are rounded to the cache's type
// for the second product (at most half a unit in the last place of each, like the rounding of the
// output); the sum is that of the rounded weights, so that they add up to one exactly as they are used.
#include "kv_internal.cuh"

namespace lif {
namespace {

struct AttendArgs {
  const void* q;
  void* out;
  float scale_log2;            // scale * log2(e): weights are powers of two
  int layer;
};

// What a stage of the ring holds.
struct __align__(16) StageInfo {
  int b, tokens, news, k0;     // place, its tokens, its new ones, first key
  int head, row0, flags;       // key-value head, first row of the row block
  int cut;                     // the item's first CTA, its last one << 16
};
enum { kOpens = 1, kStarts = 2, kEnds = 4, kCloses = 8 };   // first tile of a piece, of the item; last tile of the item, of a piece

__device__ __forceinline__ void ldm_x4(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm_x4_trans(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma(__half, float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(__nv_bfloat16, float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// a box of the pool at {column, row in the page, operand and head, page, layer}
__device__ __forceinline__ void tensor_g2s(uint32_t to, const CUtensorMap* map, int x, int row, int head, int page,
                                           int layer, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5,%6}], [%7];"
      ::"r"(to), "l"(map), "r"(x), "r"(row), "r"(head), "r"(page), "r"(layer), "r"(smem_u32(bar))
      : "memory");
}

// Byte where 16-byte piece c0 + b (c0 even and known, b 0 or 1) of row r lies in a tile of 64 rows of D
// elements: 64 columns after 64, the rest behind them; within 128 (64, 32) bytes of a row
// the pieces are permuted by the row as the tensor map's swizzle does it.
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c0, int b) {
  if (c0 / 8 < D / 64) return (c0 / 8) * 8192 + r * 128 + (((c0 & 7) ^ (b ^ (r & 7))) << 4);
  if (D % 64 == 16) return D / 64 * 8192 + r * 32 + ((b ^ (r >> 2 & 1)) << 4);
  return D / 64 * 8192 + r * 64 + (((c0 & 3) ^ (b ^ (r >> 1 & 3))) << 4);
}

template <int D, int WR, int WK>
struct Shape {
  static constexpr int kRows = 16 * WR, kWarps = WR * WK;
  static constexpr int kThreads = 32 * (kWarps + 1);                     // and one warp that loads
  static constexpr int kTileBytes = kKvTile * D * 2, kStage = 2 * kTileBytes;   // keys, or values; both
  static constexpr int kPitch = 2 * D + 16;                              // of query rows: ldmatrix without conflicts
  static constexpr int kQuerySlot = kRows * kPitch;                      // two: the next head's arrive meanwhile
  static constexpr int kTiles = D / 8;                                   // 8-column tiles of the output
  // the sum over the WK warps of a row: half of the tiles that a warp sums at a time
  static constexpr int kOwn = (kTiles + WK - 1) / WK, kPart = WK > 1 ? (kOwn + 1) / 2 : 0;
  static constexpr int kSumBytes = kWarps * kPart * 512, kJoinBytes = kWarps * 32 * 24;
  static constexpr int kScratch = kSumBytes > kJoinBytes ? kSumBytes : kJoinBytes;
  static constexpr int kMaxStages = 6;
  static constexpr int kFixed = 2 * kQuerySlot + kScratch + kRows * WK * 8 + kMaxStages * (int)sizeof(StageInfo) + 256;
  // Two CTAs an SM where three stages fit twice: one computes while the other waits.
  static constexpr int kTwo = (113 * 1024 - kFixed) / kStage, kOne = (227 * 1024 - kFixed) / kStage;
  static constexpr int kCtas = kTwo >= 3 && kWarps <= 4 ? 2 : 1;
  static constexpr int kWanted = kCtas == 2 ? kTwo : kOne;
  static constexpr int kStages = kWanted > kMaxStages ? kMaxStages : kWanted;
  static constexpr int kSmem = kStages * kStage + kFixed;
  static_assert(kStages >= 2 && kStage % 1024 == 0, "");
};

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

struct Barriers {
  uint64_t full[6], empty[6], q_empty[2], all;
  int last;                     // the CTA's answer to "is this the last piece?"
};

// The warp that loads.  Waits only for stages and query slots that the other warps have used.
template <typename T, int D, int WR, int WK>
__device__ __forceinline__ void feed(const KvMaps& maps, const KvView& V, const AttendArgs& a, unsigned char* ring,
                                     unsigned char* queries, StageInfo* info, Barriers* bars, int g0, int n_tiles,
                                     int per_cta) {
  using S = Shape<D, WR, WK>;
  constexpr int kChunks = (D + 63) / 64;
  const int lane = threadIdx.x & 31;
  const int page_tokens = 1 << V.page_shift, box = min(page_tokens, kKvTile);
  const int pages_a_tile = kKvTile / box;
  Cursor at;
  {
    const int4 p = V.cta_plan[blockIdx.x];
    at.enter(V, p.x, p.z, p.w);
    const int in = g0 - p.y, item = in / at.tiles;
    at.tile = in - item * at.tiles;
    at.head = item / at.blocks;
    at.block = item - at.head * at.blocks;
  }
  int held_b = -1, held_from = 0, held = 0;          // 32 page ids of a place, one a lane
  int stage = 0, piece = 0;
  unsigned turn = 0;
  bool lost = false;
  int i = 0;
  for (; i < n_tiles; ++i) {
    const int k0 = (at.first_tile + at.tile) * kKvTile, j0 = k0 >> V.page_shift;
    const int pages = kv_pages_of(at.tokens, V.page_shift), n_pages = min(pages - j0, pages_a_tile);
    if (at.b != held_b || (j0 & ~31) != held_from) {
      held_b = at.b;
      held_from = j0 & ~31;
      held = held_from + lane < pages ? V.table[(size_t)at.b * V.max_pages + held_from + lane] : 0;
    }
    const bool opens = i == 0 || at.tile == 0;
    if (!mbar_wait(bars->empty + stage, turn ^ 1)) lost = true;
    if (opens && !mbar_wait(bars->q_empty + (piece & 1), (piece >> 1 & 1) ^ 1)) lost = true;
    if (__any_sync(~0u, lost)) break;
    const int row0 = at.block * S::kRows, rows = min(S::kRows, at.news * V.group - row0);
    uint64_t* bar = bars->full + stage;
    if (lane == 0) {
      const int s = g0 + i - at.tile, ends = at.tile + 1 == at.tiles;
      StageInfo n;
      n.b = at.b;
      n.tokens = at.tokens;
      n.news = at.news;
      n.k0 = k0;
      n.head = at.head;
      n.row0 = row0;
      n.flags = (opens ? kOpens : 0) | (at.tile == 0 ? kStarts : 0) | (ends ? kEnds : 0) |
                (ends || i + 1 == n_tiles ? kCloses : 0);
      n.cut = opens ? s / per_cta | (s + at.tiles - 1) / per_cta << 16 : 0;
      info[stage] = n;
      mbar_expect_tx(bar, n_pages * box * D * 4 + (opens ? rows * D * 2 : 0));
    }
    __syncwarp();
    const uint32_t keys = smem_u32(ring) + stage * S::kStage;
#pragma unroll 1
    for (int x0 = 0; x0 < n_pages * 2 * kChunks; x0 += 32) {
      const int x = x0 + lane, p = x / (2 * kChunks), what = x / kChunks & 1, chunk = x % kChunks;
      const int page = __shfl_sync(~0u, held, j0 - held_from + p & 31);
      if (p < n_pages) {
        const bool full = D % 64 == 0 || chunk < D / 64;
        tensor_g2s(keys + what * S::kTileBytes + chunk * 8192 + p * box * (full ? 128 : D % 64 * 2),
                   full ? &maps.wide : &maps.rest, chunk * 64, k0 & (page_tokens - 1), what * V.n_kv_heads + at.head, page,
                   a.layer, bar);
      }
    }
    if (opens) {
      unsigned char* slot = queries + (piece & 1) * S::kQuerySlot;
      for (int r = lane; r < rows; r += 32) {
        const int t = (row0 + r) / V.group, h = row0 + r - t * V.group;
        bulk_g2s(slot + r * S::kPitch,
                 reinterpret_cast<const T*>(a.q) + (((int64_t)at.b * V.max_new + t) * V.n_heads + at.head * V.group + h) * D,
                 D * 2, bar);
      }
      ++piece;
    }
    if (++stage == S::kStages) stage = 0, turn ^= 1;
    at.step(V);
  }
  if (lost && lane == 0) flag_timeout(V.counts + LIF_KV_CNT_STATUS);
  // nobody leaves while copies are on their way
  for (int k = 0; k < min(i, S::kStages); ++k) {
    if (stage == 0) turn ^= 1;
    stage = stage == 0 ? S::kStages - 1 : stage - 1;
    mbar_wait(bars->full + stage, turn);
  }
}

// What of a cut head's row the pieces hold: the CTA's threads take four columns each, `groups` of them
// the same ones of every groups-th piece.
template <typename T, int D, int WR, int WK, typename Sync>
__device__ __forceinline__ bool join(const KvView& V, const AttendArgs& a, const StageInfo& at, int rows, int first, int pieces,
                                     unsigned char* scratch, Sync sync) {
  using S = Shape<D, WR, WK>;
  constexpr int kN = S::kWarps * 32;
  const size_t slot = (size_t)S::kRows * (D + 2);
  const int units = rows * (D / 4);
  int groups = 1;
  while (groups < 8 && 2 * groups * units <= kN && groups < pieces) groups *= 2;
  float4* outs = reinterpret_cast<float4*>(scratch);
  float2* tops = reinterpret_cast<float2*>(scratch + kN * 16);
  for (int u = threadIdx.x; u < (groups > 1 ? kN : units); u += kN) {
    const int group = u / units, unit = u - group * units, r = unit / (D / 4), c = unit % (D / 4);
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (group < groups) {
      for (int p0 = group; p0 < pieces; p0 += 8 * groups) {
        float pm[8], pl[8];
        float4 x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int p = p0 + e * groups;
          pm[e] = -INFINITY;
          pl[e] = 0.f;
          x[e] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (p < pieces) {                        // piece p: the first CTA's second slot, every other one's first
            const float* from = V.partials + (size_t)(2 * (first + p) + (p == 0)) * slot;
            pm[e] = __ldcg(from + S::kRows * D + r);
            pl[e] = __ldcg(from + S::kRows * (D + 1) + r);
            x[e] = __ldcg(reinterpret_cast<const float4*>(from + (size_t)r * D) + c);
          }
        }
        float top = m;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, pm[e]);
        const float base = top == -INFINITY ? 0.f : top, shrink = exp2f(m - base);
        m = top;
        l *= shrink;
        acc = make_float4(acc.x * shrink, acc.y * shrink, acc.z * shrink, acc.w * shrink);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = exp2f(pm[e] - base);
          l = fmaf(pl[e], w, l);
          acc.x = fmaf(w, x[e].x, acc.x);
          acc.y = fmaf(w, x[e].y, acc.y);
          acc.z = fmaf(w, x[e].z, acc.z);
          acc.w = fmaf(w, x[e].w, acc.w);
        }
      }
    }
    if (groups > 1) {                              // (every thread is here, once)
      outs[u] = acc;
      tops[u] = make_float2(m, l);
      if (!sync()) return false;
      if (group == 0) {
        float top = m;
        for (int k = 1; k < groups; ++k) top = fmaxf(top, tops[u + k * units].x);
        const float base = top == -INFINITY ? 0.f : top;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
        for (int k = 0; k < groups; ++k) {
          const float2 t = tops[u + k * units];
          const float4 x = outs[u + k * units];
          const float w = exp2f(t.x - base);
          l = fmaf(t.y, w, l);
          sum.x = fmaf(w, x.x, sum.x);
          sum.y = fmaf(w, x.y, sum.y);
          sum.z = fmaf(w, x.z, sum.z);
          sum.w = fmaf(w, x.w, sum.w);
        }
        acc = sum;
      }
    }
    if (group == 0) {
      const int t = (at.row0 + r) / V.group, h = at.row0 + r - t * V.group;
      T* to = reinterpret_cast<T*>(a.out) + (((int64_t)at.b * V.max_new + t) * V.n_heads + at.head * V.group + h) * D + 4 * c;
      *reinterpret_cast<uint2*>(to) = make_uint2(Num<T>::from2(acc.x / l, acc.y / l), Num<T>::from2(acc.z / l, acc.w / l));
    }
  }
  return groups == 1 || sync();                    // the scratch is free again
}

template <typename T, int D, int WR, int WK>
__global__ void __launch_bounds__(Shape<D, WR, WK>::kThreads, Shape<D, WR, WK>::kCtas)
kv_attention_kernel(const __grid_constant__ KvMaps maps, KvView V, AttendArgs a) {
  using S = Shape<D, WR, WK>;
  constexpr int kSteps = D / 16;                     // k steps of the first product
  constexpr int kKeys = kKvTile / WK, kNT = kKeys / 8;   // a warp's keys of a tile
  constexpr int kTiles = S::kTiles;
  constexpr bool kHold = D <= 128;                   // the rows' queries stay in registers
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* queries = smem + S::kStages * S::kStage;
  unsigned char* scratch = queries + 2 * S::kQuerySlot;
  float2* stats = reinterpret_cast<float2*>(scratch + S::kScratch);            // [rows][WK] maximum, sum
  StageInfo* info = reinterpret_cast<StageInfo*>(scratch + S::kScratch + S::kRows * WK * 8);
  Barriers* bars = reinterpret_cast<Barriers*>(info + S::kMaxStages);
  static_assert(sizeof(Barriers) <= 256, "");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(bars->full + i, 1);
      mbar_init(bars->empty + i, S::kWarps);
    }
    mbar_init(bars->q_empty, S::kWarps);
    mbar_init(bars->q_empty + 1, S::kWarps);
    mbar_init(&bars->all, S::kWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int total = V.counts[KV_TILES], per_cta = V.counts[KV_TILES_PER_CTA];
  const int g0 = blockIdx.x * per_cta;
  if (g0 >= total) return;
  const int n_tiles = min(total - g0, per_cta);
  if (warp == S::kWarps) {
    feed<T, D, WR, WK>(maps, V, a, smem, queries, info, bars, g0, n_tiles, per_cta);
    return;
  }

  const int wr = warp / WK, wk = warp % WK;
  unsigned syncs = 0;
  auto sync = [&]() {                                // the warps that compute; bounded as every wait
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->all);
    return mbar_wait(&bars->all, syncs++ & 1);
  };
  auto release = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  float o[kTiles][4];                  // rows g, g + 8; all columns
  float m[2], sum[2];                  // running maximum; this lane's share of the sum
  int upto[2];                         // last key that the row sees
  uint32_t qf[kHold ? kSteps : 1][4];
  int stage = 0, slot = -1, rows = 0, cut = 0;
  bool starts = false, idle = false;
  unsigned turn = 0;
  const uint32_t ring = smem_u32(smem), q_lane = smem_u32(queries) + (wr * 16 + (lane & 15)) * S::kPitch + (lane >> 4) * 16;
  const int key_row = wk * kKeys + (lane & 7) + (lane >> 4) * 8, key_b = lane >> 3 & 1;
  const int val_row = wk * kKeys + (lane & 15), val_b = lane >> 4;
#pragma unroll 1
  for (int i = 0; i < n_tiles; ++i) {
    if (!mbar_wait(bars->full + stage, turn)) {
      if (lane == 0) flag_timeout(V.counts + LIF_KV_CNT_STATUS);
      return;
    }
    const StageInfo at = info[stage];
    if (at.flags & kOpens) {           // another head's rows
      slot ^= 1;
      if (slot < 0) slot = 0;
      starts = at.flags & kStarts;
      cut = at.cut;
      rows = min(S::kRows, at.news * V.group - at.row0);
      idle = WR > 1 && wr * 16 >= rows;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = (at.row0 + wr * 16 + g + 8 * h) / V.group;
        upto[h] = at.tokens - at.news + min(t, at.news - 1);
        m[h] = -INFINITY;
        sum[h] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < kTiles; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      if (kHold) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) ldm_x4(qf[k], q_lane + slot * S::kQuerySlot + k * 32);
        release(bars->q_empty + slot);
      }
    }
    const uint32_t keys = ring + stage * S::kStage, values = keys + S::kTileBytes;
    if (!idle) {
      float s[kNT][4];
#pragma unroll
      for (int n = 0; n < kNT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        uint32_t qa[4];
        if (!kHold) ldm_x4(qa, q_lane + slot * S::kQuerySlot + k * 32);
#pragma unroll
        for (int n = 0; n < kNT; n += 2) {
          uint32_t kf[4];
          ldm_x4(kf, keys + piece<D>(key_row + n * 8, 2 * k, key_b));
          mma(T(), s[n], kHold ? qf[k] : qa, kf[0], kf[1]);
          mma(T(), s[n + 1], kHold ? qf[k] : qa, kf[2], kf[3]);
        }
      }
      // keys that not every row sees
      const int lowest = kv_first_key(at.tokens, at.news, V.window);
      const bool edge = at.k0 + kKvTile > at.tokens - at.news + 1 || (V.window > 0 && at.k0 <= at.tokens - 1 - V.window);
      const int reach = V.window > 0 ? V.window : 0x7fffffff;
      const int first = at.k0 + wk * kKeys;
#pragma unroll
      for (int n = 0; n < kNT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] *= a.scale_log2;
      if (edge) {
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = first + n * 8 + 2 * t4 + (e & 1), last = upto[e >> 1];
            if (key > last || last - key >= reach) s[n][e] = -INFINITY;
          }
      }
      // weights 2^(s - max); a row that has seen nothing yet keeps max = -inf and weights 0
      uint32_t w[kNT][2];
      float shrink[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = m[h];
#pragma unroll
        for (int n = 0; n < kNT; ++n) top = fmaxf(top, fmaxf(s[n][2 * h], s[n][2 * h + 1]));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        const float base = top == -INFINITY ? 0.f : top;
        shrink[h] = exp2f(m[h] - base);
        m[h] = top;
        float add = 0.f;
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          w[n][h] = Num<T>::from2(exp2f(s[n][2 * h] - base), exp2f(s[n][2 * h + 1] - base));
          const float2 used = Num<T>::to2(w[n][h]);
          add += used.x + used.y;
        }
        sum[h] = fmaf(sum[h], shrink[h], add);
      }
      if (__any_sync(~0u, shrink[0] != 1.f || shrink[1] != 1.f)) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          o[j][0] *= shrink[0];
          o[j][1] *= shrink[0];
          o[j][2] *= shrink[1];
          o[j][3] *= shrink[1];
        }
      }
      // A row's weight of a key that it does not see is 0, but 0 times an infinite or NaN value is not.
      // Values that no row sees are cleared; where rows differ in what they see and a value is not
      // finite, the products are formed one by one, the unseen ones left out.
      bool one_by_one = false;
      if (edge) {
        bool odd = false;
#pragma unroll 1
        for (int x = lane; x < kKeys * (D / 8); x += 32) {
          const int r = wk * kKeys + x / (D / 8), c = x % (D / 8), key = at.k0 + r;
          uint4* v = reinterpret_cast<uint4*>(smem + (values - ring) + (c / 8 < D / 64 ? (c / 8) * 8192 + r * 128 + ((c & 7) ^ (r & 7)) * 16
                                                                       : D % 64 == 16 ? D / 64 * 8192 + r * 32 + ((c & 1) ^ (r >> 2 & 1)) * 16
                                                                                      : D / 64 * 8192 + r * 64 + ((c & 3) ^ (r >> 1 & 3)) * 16));
          if (key >= at.tokens || key < lowest) {
            *v = make_uint4(0, 0, 0, 0);
          } else if (at.news > 1) {
            const uint4 bits = *v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t y = (&bits.x)[e], lo = Num<T>::kExponent & 0xffffu, hi = Num<T>::kExponent & 0xffff0000u;
              odd = odd || (y & lo) == lo || (y & hi) == hi;
            }
          }
        }
        one_by_one = __any_sync(~0u, odd);
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the ring's copies come behind these stores
      }
      if (!one_by_one) {
#pragma unroll
        for (int n = 0; n < kNT; n += 2) {
          const uint32_t wf[4] = {w[n][0], w[n][1], w[n + 1][0], w[n + 1][1]};
#pragma unroll
          for (int j = 0; j < kTiles; j += 2) {
            uint32_t vf[4];
            ldm_x4_trans(vf, values + piece<D>(val_row + n * 8, j, val_b));
            mma(T(), o[j], wf, vf[0], vf[1]);
            mma(T(), o[j + 1], wf, vf[2], vf[3]);
          }
        }
      } else {
#pragma unroll 1
        for (int k = 0; k < kKeys; ++k) {
          uint32_t pair[2] = {w[0][0], w[0][1]};
#pragma unroll
          for (int n = 1; n < kNT; ++n)
            if (k >> 3 == n) pair[0] = w[n][0], pair[1] = w[n][1];
          float wt[2];
          bool sees[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 x = Num<T>::to2(__shfl_sync(~0u, pair[h], (lane & 28) + (k >> 1 & 3)));
            wt[h] = k & 1 ? x.y : x.x;
            sees[h] = first + k <= upto[h] && upto[h] - (first + k) < reach;
          }
          const int r = wk * kKeys + k;
#pragma unroll
          for (int j = 0; j < kTiles; ++j) {
            const float2 v = Num<T>::to2(*reinterpret_cast<const uint32_t*>(
                smem + (values - ring) + piece<D>(r, j & ~1, j & 1) + 4 * t4));
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (sees[h]) {
                o[j][2 * h] = fmaf(wt[h], v.x, o[j][2 * h]);
                o[j][2 * h + 1] = fmaf(wt[h], v.y, o[j][2 * h + 1]);
              }
          }
        }
      }
    }
    release(bars->empty + stage);
    if (++stage == S::kStages) stage = 0, turn ^= 1;

    if (at.flags & kCloses) {
      if (!kHold) release(bars->q_empty + slot);
      float all[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        all[h] = sum[h] + __shfl_xor_sync(~0u, sum[h], 1);
        all[h] += __shfl_xor_sync(~0u, all[h], 2);
      }
      if constexpr (WK > 1) {
        // the row's WK warps: a common maximum, then every warp sums its share of the columns
        if (t4 == 0) {
#pragma unroll
          for (int h = 0; h < 2; ++h) stats[(wr * 16 + g + 8 * h) * WK + wk] = make_float2(m[h], all[h]);
        }
        if (!sync()) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float2 x[WK];
          float top = -INFINITY;
#pragma unroll
          for (int k = 0; k < WK; ++k) {
            x[k] = stats[(wr * 16 + g + 8 * h) * WK + k];
            top = fmaxf(top, x[k].x);
          }
          const float base = top == -INFINITY ? 0.f : top, shrink = exp2f(m[h] - base);
          all[h] = 0.f;
#pragma unroll
          for (int k = 0; k < WK; ++k) all[h] = fmaf(x[k].y, exp2f(x[k].x - base), all[h]);
          m[h] = top;
#pragma unroll
          for (int j = 0; j < kTiles; ++j) {
            o[j][2 * h] *= shrink;
            o[j][2 * h + 1] *= shrink;
          }
        }
        float4* box = reinterpret_cast<float4*>(scratch);
#pragma unroll 1
        for (int k = 1; k < WK; ++k) {
          const int other = (wk + k) % WK;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (half * S::kPart >= S::kOwn) continue;
            if ((k > 1 || half) && !sync()) return;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
              const int in = j / WK - half * S::kPart;
              if (in >= 0 && in < S::kPart && j % WK == other && !idle)
                box[((wr * WK + other) * S::kPart + in) * 32 + lane] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
            }
            if (!sync()) return;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
              const int in = j / WK - half * S::kPart;
              if (in >= 0 && in < S::kPart && j % WK == wk && !idle) {
                const float4 x = box[(warp * S::kPart + in) * 32 + lane];
                o[j][0] += x.x;
                o[j][1] += x.y;
                o[j][2] += x.z;
                o[j][3] += x.w;
              }
            }
          }
        }
      }
      const bool whole = starts && (at.flags & kEnds);
      // a piece that began before this CTA's run, or one that goes on behind it
      float* part = V.partials + (size_t)(2 * blockIdx.x + starts) * S::kRows * (D + 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = wr * 16 + g + 8 * h;
        if (r >= rows) continue;
        if (whole) {
          const int t = (at.row0 + r) / V.group, head = at.head * V.group + at.row0 + r - t * V.group;
          T* out = reinterpret_cast<T*>(a.out) + (((int64_t)at.b * V.max_new + t) * V.n_heads + head) * D;
          const float inv = 1.f / all[h];
#pragma unroll
          for (int j = 0; j < kTiles; ++j)
            if (j % WK == wk)
              *reinterpret_cast<uint32_t*>(out + j * 8 + 2 * t4) = Num<T>::from2(o[j][2 * h] * inv, o[j][2 * h + 1] * inv);
        } else {
#pragma unroll
          for (int j = 0; j < kTiles; ++j)
            if (j % WK == wk) *reinterpret_cast<float2*>(part + (size_t)r * D + j * 8 + 2 * t4) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
          if (wk == 0 && t4 == 0) {
            part[S::kRows * D + r] = m[h];
            part[S::kRows * (D + 1) + r] = all[h];
          }
        }
      }
      if (!whole) {
        const int from = cut & 0xffff, pieces = (cut >> 16) - from + 1;
        __threadfence();
        if (!sync()) return;
        if (threadIdx.x == 0) {
          const int before = atomicAdd(V.tickets + from, 1);
          bars->last = before == pieces - 1;
          if (bars->last) V.tickets[from] = 0;
          __threadfence();
        }
        if (!sync()) return;
        if (bars->last) {
          __threadfence();
          if (!join<T, D, WR, WK>(V, a, at, rows, from, pieces, scratch, sync)) return;
        }
      }
    }
  }
}

// What to do with the kernel for a type, head dimension and row tiles: few rows leave the tile's keys to more warps.
template <typename T, int D, int WR, int WK, typename F>
cudaError_t with(F f) {
  using S = Shape<D, WR, WK>;
  return f(kv_attention_kernel<T, D, WR, WK>, S::kThreads, S::kSmem);
}
template <typename T, int D, typename F>
cudaError_t with_rows(int row_tiles, F f) {
  if (row_tiles == 1) return with<T, D, 1, 4>(f);
  if constexpr (D <= 128) {
    if (row_tiles == 2) return with<T, D, 2, 4>(f);
    if (row_tiles == 4) return with<T, D, 4, 2>(f);
    return with<T, D, 8, 1>(f);
  } else {                               // 128 registers of output: four warps that compute
    if (row_tiles == 2) return with<T, D, 2, 2>(f);
    return with<T, D, 4, 1>(f);
  }
}
template <typename T, typename F>
cudaError_t with_dim(int dim, int row_tiles, F f) {
  switch (dim) {
    case 64: return with_rows<T, 64>(row_tiles, f);
    case 80: return with_rows<T, 80>(row_tiles, f);
    case 96: return with_rows<T, 96>(row_tiles, f);
    case 128: return with_rows<T, 128>(row_tiles, f);
    default: return with_rows<T, 256>(row_tiles, f);
  }
}
template <typename F>
cudaError_t with_kernel(const lif_kv* kv, F f) {
  const lif_kv_desc& d = kv->desc;
  return d.dtype == LIF_TYPE_F16 ? with_dim<__half>(d.head_dim, kv->row_tiles, f)
                                 : with_dim<__nv_bfloat16>(d.head_dim, kv->row_tiles, f);
}

// The pool as the tensor copies see it: a box is `columns` wide and as many rows as a tile takes of a page.
bool encode_map(CUtensorMap* map, const lif_kv_desc& d, int columns, CUtensorMapSwizzle swizzle) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  void* entry = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &entry, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess || !entry)
    return false;
  const cuuint64_t D = d.head_dim, P = d.page_tokens, heads = 2 * (cuuint64_t)d.n_kv_heads;
  const cuuint64_t dims[5] = {D, P, heads, (cuuint64_t)d.n_pages, (cuuint64_t)d.n_layers};
  const cuuint64_t strides[4] = {D * 2, P * D * 2, heads * P * D * 2, (cuuint64_t)d.n_pages * heads * P * D * 2};
  const cuuint32_t box[5] = {(cuuint32_t)columns, (cuuint32_t)(P < kKvTile ? P : kKvTile), 1, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return reinterpret_cast<Encode>(entry)(
             map, d.dtype == LIF_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, d.dev_pages,
             dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

// Smallest block of rows that holds a key-value head's rows of one sequence, so that its keys are
// read once, up to what registers and shared memory take (128 rows, 64 at 256 columns).
int kv_row_tiles(const lif_kv_desc& d) {
  const int rows = d.n_heads / d.n_kv_heads * d.max_new, most = d.head_dim <= 128 ? 8 : 4;
  int t = 1;
  while (t < most && t * 16 < rows) t *= 2;
  return t;
}

bool kv_attention_configure(lif_kv* kv, int* ctas_per_sm) {
  const int rest = kv->desc.head_dim % 64;
  if (!encode_map(&kv->maps.wide, kv->desc, 64, CU_TENSOR_MAP_SWIZZLE_128B)) return false;
  if (rest && !encode_map(&kv->maps.rest, kv->desc, rest, rest == 16 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_64B))
    return false;
  return with_kernel(kv, [&](auto kernel, int threads, int smem) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, kernel, threads, smem);
    return e;
  }) == cudaSuccess;
}

cudaError_t launch_kv_attention(const lif_kv* kv, int layer, const void* q, void* out, cudaStream_t st) {
  AttendArgs a;
  a.q = q;
  a.out = out;
  a.scale_log2 = kv->scale * 1.4426950408889634f;
  a.layer = layer;
  return with_kernel(kv, [&](auto kernel, int threads, int smem) {
    return launch_k2(kernel, dim3(kv->v.ctas), dim3(threads), smem, st, 1, 1, kv->maps, kv->v, a);
  });
}

}  // namespace lif
