// Attention of a step's new tokens over the paged key-value cache.
//
//   out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale <q_row, k_j> - max_j)
//
// Rows: the new tokens' query heads that share a key-value head, `group` x tokens of them (1 .. 16
// mostly), in blocks of 16 x WR (more than 16 rows of 64 or 128 elements: kv_attention_wide.cu).  Every key and
// value is read once per row block; bound: HBM (64 sequences of 300 .. 4000 under 56 heads of 128: 2.5 GB in 359 us,
// 1.05 of measured; 8 ragged ones: 59 us, 94%), and latency where the step is small: one sequence of 1000 under 32
// heads takes 7.6 us, 2.5 of them its bytes (table and plan 1, first copy 1, two tiles 1.6, their sum 0.6, join 2.4).
//
// Split.  The step's work is numbered in tiles of 64 keys (kv_plan) and cut into runs, across heads and
// sequences, so that one long sequence, many short ones and anything ragged between fill the chip alike.
// Every CTA begins with a run of its own; where the work is long these cover most of it and the
// rest is taken in short runs by whoever is free: CTAs with equal work differ by a fifth in time (memory is nearer to
// some pages than to others), and 64 sequences of 56 heads went from 451 to 360 us.  A head that a run's end cuts is
// finished by kv_join_kernel from the pieces' {reference, sum, unnormalised output}.  Which run holds which tiles
// does not depend on who takes it, and pieces are joined in their order: the same bits every time.
//
// Loads.  One warp feeds the others: it walks the run, reads 32 page ids at a time and moves keys and
// values into a ring of stages with tensor copies (TMA), a copy per page, 64 columns and operand, which
// store a row's 16-byte pieces in the permuted order that makes ldmatrix free of bank conflicts.  What a
// stage holds (place, head, first key ...) travels beside it, so the other warps divide nothing.
// Tokens past the end lie in the same page and are copied too; the values among them are cleared in
// shared memory before use (whatever they hold, 0 times it is not 0), the scores replaced by -inf.
//
// Products.  Of 64 keys each of WK warps takes 64 / WK, of the rows each of WR warps 16, and keeps a
// running reference (kv_attention.cuh), sum and output of its own (mma m16n8k16): between two tiles no warp waits for another,
// and the weights stay in registers from the first product to the second.  The WK warps of a row
// are summed when the head ends.
//
// Precision.  Scores, references, sums and outputs are fp32.  Weights are rounded to the cache's type
// for the second product: at most half a unit in the last place of each, like the rounding of the
// output; in fp16, of a weight below 2^-21 of the row's largest, 2^-32 of that one.  The sum is that of
// the rounded weights, so that they add up to one exactly as they are used.
#include "kv_attention.cuh"

namespace lif {
namespace {

__device__ __forceinline__ void ldm_x4(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm_x4_trans(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma(__half, float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(__nv_bfloat16, float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int D, int WR, int WK>
struct Shape {
  static constexpr int kRows = 16 * WR, kWarps = WR * WK;
  static constexpr int kThreads = 32 * (kWarps + 1);                     // and one warp that loads
  static constexpr int kTileBytes = kKvTile * D * 2, kStage = 2 * kTileBytes;   // keys, or values; both
  static constexpr bool kHold = D <= 128;                                // queries stay in registers while a head lasts
  // Many rows come a copy per token, one behind the other, which the one ldmatrix of each pays for with
  // conflicts; few rows, or rows read for every tile, a copy per row, 16 bytes apart.
  static constexpr bool kDense = kHold && WR > 1;
  static constexpr int kPitch = kDense ? 2 * D : 2 * D + 16;
  static constexpr int kQuerySlot = kRows * kPitch;                      // two: the next head's arrive meanwhile
  static constexpr int kTiles = D / 8;                                   // 8-column tiles of the output
  // the sum over the WK warps of a row: so many of a warp's rows at a time
  static constexpr int kSumRows = WR > 1 || D == 96 ? 4 : D < 96 ? 8 : 2, kSumPitch = D + 8;
  static constexpr int kScratch = WK > 1 ? kWarps * kSumRows * kSumPitch * 4 : 0;
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

struct Barriers {
  uint64_t full[6], empty[6], q_empty[2], all;
};

// The warp that loads.  Waits only for stages and query slots that the other warps have used.
template <typename T, int D, int WR, int WK>
__device__ __forceinline__ void feed(const KvMaps& maps, const KvView& V, const AttendArgs& a, unsigned char* ring,
                                     unsigned char* queries, StageInfo* info, Barriers* bars, int4 plan, int4 step) {
  using S = Shape<D, WR, WK>;
  constexpr bool kLinear = D == 80;                  // a page's rows of a head as they are
  constexpr int kChunks = kLinear ? 1 : (D + 63) / 64;
  const int lane = threadIdx.x & 31;
  const int page_tokens = 1 << V.page_shift, box = min(page_tokens, kKvTile);
  Walk walk(V, blockIdx.x, plan, step);
  const Cursor& at = walk.at;
  int stage = 0, piece = 0;
  unsigned turn = 0;
  bool lost = false;
  int i = 0;
  for (; !walk.last; ++i) {
    walk.begin(V, lane);
    const bool opens = walk.opens;
    const int k0 = walk.k0, n_pages = walk.n_pages;
    if (!mbar_wait(bars->empty + stage, turn ^ 1)) lost = true;
    if (opens && !mbar_wait(bars->q_empty + (piece & 1), (piece >> 1 & 1) ^ 1)) lost = true;
    if (__any_sync(~0u, lost)) break;                // (nothing of this tile is on its way)
    const int row0 = at.block * S::kRows, rows = min(S::kRows, at.news * V.group - row0);
    uint64_t* bar = bars->full + stage;
    if (lane == 0) {
      info[stage] = walk.info(V);
      mbar_expect_tx(bar, n_pages * box * D * 4 + (opens ? rows * D * 2 : 0));
    }
    __syncwarp();
    const uint32_t keys = smem_u32(ring) + stage * S::kStage;
#pragma unroll 1
    for (int x0 = 0; x0 < n_pages * 2 * kChunks; x0 += 32) {
      const int x = x0 + lane, p = x / (2 * kChunks), what = x / kChunks & 1, chunk = x % kChunks;
      const int page = __shfl_sync(~0u, walk.held, walk.j0 - walk.held_from + p & 31);
      if (kLinear && p < n_pages) {
        const int64_t head = ((int64_t)page * 2 + what) * V.n_kv_heads + at.head;
        bulk_g2s(ring + stage * S::kStage + what * S::kTileBytes + p * box * D * 2,
                 reinterpret_cast<const T*>(a.pages) + ((head << V.page_shift) + (k0 & (page_tokens - 1))) * D, box * D * 2, bar);
      } else if (p < n_pages) {
        const bool full = D % 64 == 0 || chunk < D / 64;
        tensor_g2s(keys + what * S::kTileBytes + chunk * 8192 + p * box * (full ? 128 : 64),
                   full ? &maps.wide : &maps.rest, chunk * 64, k0 & (page_tokens - 1), what * V.n_kv_heads + at.head, page,
                   a.layer, bar);
      }
    }
    if (opens) {
      unsigned char* slot = queries + (piece & 1) * S::kQuerySlot;
      const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)at.b * V.max_new * V.n_heads + at.head * V.group) * D;
      const int t0 = row0 / V.group;                 // row r: head (row0 + r) % group of token (row0 + r) / group
      if (S::kDense) {
        for (int t = t0 + lane; t * V.group < row0 + rows; t += 32) {
          const int r0 = max(0, t * V.group - row0), r1 = min(rows, (t + 1) * V.group - row0);
          bulk_g2s(slot + r0 * S::kPitch, q + ((int64_t)t * V.n_heads + row0 + r0 - t * V.group) * D, (r1 - r0) * D * 2, bar);
        }
      } else {
        for (int r = lane; r < rows; r += 32) {
          const int t = (row0 + r) / V.group;
          bulk_g2s(slot + r * S::kPitch, q + ((int64_t)t * V.n_heads + row0 + r - t * V.group) * D, D * 2, bar);
        }
      }
      ++piece;
    }
    if (++stage == S::kStages) stage = 0, turn ^= 1;
    walk.advance(V);
  }
  if (lost && lane == 0) flag_timeout(V.counts + LIF_KV_CNT_STATUS);
  // nobody leaves while copies are on their way
  for (int k = 0; k < min(i, S::kStages); ++k) {
    if (stage == 0) turn ^= 1;
    stage = stage == 0 ? S::kStages - 1 : stage - 1;
    mbar_wait(bars->full + stage, turn);
  }
}

template <typename T, int D, int WR, int WK>
__global__ void __launch_bounds__(Shape<D, WR, WK>::kThreads, Shape<D, WR, WK>::kCtas)
kv_attention_kernel(const __grid_constant__ KvMaps maps, KvView V, AttendArgs a) {
  using S = Shape<D, WR, WK>;
  constexpr int kSteps = D / 16;                     // k steps of the first product
  constexpr int kKeys = kKvTile / WK, kNT = kKeys / 8;   // a warp's keys of a tile
  constexpr int kTiles = S::kTiles;
  constexpr bool kHold = S::kHold;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* queries = smem + S::kStages * S::kStage;
  unsigned char* scratch = queries + 2 * S::kQuerySlot;
  float2* stats = reinterpret_cast<float2*>(scratch + S::kScratch);            // [rows][WK] reference, sum
  StageInfo* info = reinterpret_cast<StageInfo*>(scratch + S::kScratch + S::kRows * WK * 8);
  Barriers* bars = reinterpret_cast<Barriers*>(info + S::kMaxStages);
  static_assert(sizeof(Barriers) <= 256, "");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.wide) : "memory");
    if (D == 96) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.rest) : "memory");
  }
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
  const int4 plan = V.run_plan[blockIdx.x], step = *reinterpret_cast<const int4*>(V.counts + KV_TILES);
  if (blockIdx.x >= step.y) return;
  if (warp == S::kWarps) {
    feed<T, D, WR, WK>(maps, V, a, smem, queries, info, bars, plan, step);
    return;
  }

  const int wr = warp / WK, wk = warp % WK;
  unsigned syncs = 0;
  auto sync = [&]() {                                // the warps that compute; bounded as every wait
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->all);
    return (bool)__all_sync(~0u, mbar_wait(&bars->all, syncs++ & 1, 2 * kWaitLimit));   // (a warp that still waits for a tile comes, or never will)
  };
  auto release = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  float o[kTiles][4];                  // rows g, g + 8; all columns
  float m[2], sum[2];                  // what weights refer to; this lane's share of their sum
  int upto[2];                         // last key that the row sees
  uint32_t qf[kHold ? kSteps : 1][4];
  int stage = 0, slot = 1, rows = 0;
  bool starts = false, idle = false;
  unsigned turn = 0;
  const uint32_t ring = smem_u32(smem), q_lane = smem_u32(queries) + (wr * 16 + (lane & 15)) * S::kPitch + (lane >> 4) * 16;
  const int key_row = wk * kKeys + (lane & 7) + (lane >> 4) * 8, key_b = lane >> 3 & 1;
  const int val_row = wk * kKeys + (lane & 15), val_b = lane >> 4;
#pragma unroll 1
  for (bool last = false; !last;) {
    if (!__all_sync(~0u, mbar_wait(bars->full + stage, turn))) {   // (the warp's lanes go on, or give up, together)
      if (lane == 0) flag_timeout(V.counts + LIF_KV_CNT_STATUS);
      return;
    }
    const StageInfo at = info[stage];
    last = at.flags & kLast;
    if (at.flags & kOpens) {           // another head's rows
      slot ^= 1;
      starts = at.flags & kStarts;
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
      const int first = at.k0 + wk * kKeys, reach = V.window > 0 ? V.window : 0x7fffffff;
      // A row's weight of a key that it does not see is 0, but 0 times an infinite or NaN value is not.
      // Values that no row sees are cleared; where rows differ in what they see and a value is not
      // finite, the products are formed one by one, the unseen ones left out.
      bool one_by_one = false;
      if (at.flags & kEdge) {
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = first + n * 8 + 2 * t4 + (e & 1), last_seen = upto[e >> 1];
            if (key > last_seen || last_seen - key >= reach) s[n][e] = -INFINITY;
          }
        const Edge edge(V, at);
        const bool clear = edge.clear(at, first, kKeys), differ = edge.differ(at, first, kKeys);
        if (clear || differ) {
          constexpr int kPieces = D / 8, kLanes = kPieces <= 8 ? 8 : kPieces <= 16 ? 16 : 32;
          const int c = lane % kLanes;
          bool odd = false;
          for (int k = lane / kLanes; k < kKeys; k += 32 / kLanes) {
            const int r = wk * kKeys + k;
            const bool none = edge.none(at, first + k);
            if (c >= kPieces || !(none || differ)) continue;
            uint4* v = reinterpret_cast<uint4*>(smem + (values - ring) + piece<D>(r, c));
            if (none) {
              *v = make_uint4(0, 0, 0, 0);
            } else {
              odd = odd || any_not_finite<T>(*v);
            }
          }
          one_by_one = __any_sync(~0u, odd);
          __syncwarp();
          if (clear) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the ring's copies come behind these stores
        }
      }
      // weights 2^(s - m); a row that has seen nothing yet has m = -inf and weights 0
      bool above = false;
      float top[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        top[h] = fmaxf(s[0][2 * h], s[0][2 * h + 1]);
#pragma unroll
        for (int n = 1; n < kNT; ++n) top[h] = fmaxf(top[h], fmaxf(s[n][2 * h], s[n][2 * h + 1]));
        above = above || too_far<T>(top[h], a.scale_log2, m[h]);
      }
      if (__any_sync(~0u, above)) {
        float shrink[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 1));
          top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 2));
          // (each row by itself: what a row gets must not depend on the others, which may not be there)
          const float now = too_far<T>(top[h], a.scale_log2, m[h]) ? new_reference<T>(top[h], a.scale_log2) : m[h];
          shrink[h] = power(m[h] - (now == -INFINITY ? 0.f : now));
          m[h] = now;
          sum[h] *= shrink[h];
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          o[j][0] *= shrink[0];
          o[j][1] *= shrink[0];
          o[j][2] *= shrink[1];
          o[j][3] *= shrink[1];
        }
      }
      uint32_t w[kNT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float base = m[h] == -INFINITY ? 0.f : m[h];
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          w[n][h] = Num<T>::from2(power(fmaf(s[n][2 * h], a.scale_log2, -base)), power(fmaf(s[n][2 * h + 1], a.scale_log2, -base)));
          const float2 used = Num<T>::to2(w[n][h]);
          sum[h] += used.x + used.y;
        }
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
      const bool whole = starts && (at.flags & kEnds);
      // a piece that began before this run, or one that goes on behind it
      float* part = V.partials + (size_t)(2 * at.run + starts) * V.slot_floats;
      T* out = reinterpret_cast<T*>(a.out);
      if constexpr (WK > 1) {
        // The row's WK warps lay down their outputs, a few rows at a time, and each thread sums two columns.  The
        // first wait is bounded: a warp that gave up waiting for a tile is not there.  Past it all of them are.
        float* mine = reinterpret_cast<float*>(scratch) + warp * S::kSumRows * S::kSumPitch;
        const float* theirs = reinterpret_cast<const float*>(scratch) + wr * WK * S::kSumRows * S::kSumPitch;
        const int live = min(16, rows - wr * 16);
#pragma unroll 1
        for (int r0 = 0; r0 < 16; r0 += S::kSumRows) {
          if (r0 && r0 >= live) break;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h - r0;
            if (r < 0 || r >= S::kSumRows || idle) continue;
            if (t4 == 0) stats[(wr * 16 + r0 + r) * WK + wk] = make_float2(m[h], all[h]);
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
              *reinterpret_cast<float2*>(mine + r * S::kSumPitch + j * 8 + 2 * t4) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
          }
          if (r0 == 0) {
            if (!sync()) return;
          } else {
            asm volatile("bar.sync %0, %1;" ::"r"(1 + wr), "n"(32 * WK) : "memory");
          }
#pragma unroll 1
          for (int x = wk * 32 + lane; x < S::kSumRows * D / 2; x += 32 * WK) {
            const int r = x / (D / 2), c = 2 * (x - r * (D / 2)), row = wr * 16 + r0 + r;
            if (row >= rows) break;
            float2 st[WK], sum2 = make_float2(0.f, 0.f);
            float top = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < WK; ++k) {
              st[k] = stats[row * WK + k];
              top = fmaxf(top, st[k].x);
            }
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int k = 0; k < WK; ++k) {
              const float f = power(st[k].x - base);
              const float2 y = *reinterpret_cast<const float2*>(theirs + (k * S::kSumRows + r) * S::kSumPitch + c);
              l = fmaf(st[k].y, f, l);
              sum2.x = fmaf(f, y.x, sum2.x);
              sum2.y = fmaf(f, y.y, sum2.y);
            }
            if (whole) {
              *reinterpret_cast<uint32_t*>(out + row_offset(V, at, row) + c) = Num<T>::from2(sum2.x / l, sum2.y / l);
            } else {
              *reinterpret_cast<float2*>(part + (size_t)row * (D + 4) + c) = sum2;
              if (c == 0) *reinterpret_cast<float2*>(part + (size_t)row * (D + 4) + D) = make_float2(top, l);
            }
          }
          asm volatile("bar.sync %0, %1;" ::"r"(1 + wr), "n"(32 * WK) : "memory");
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = wr * 16 + g + 8 * h;
          if (r >= rows) continue;
          if (whole) {
            T* to = out + row_offset(V, at, r) + 2 * t4;
            const float inv = 1.f / all[h];
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
              *reinterpret_cast<uint32_t*>(to + j * 8) = Num<T>::from2(o[j][2 * h] * inv, o[j][2 * h + 1] * inv);
          } else {
            float* to = part + (size_t)r * (D + 4);
#pragma unroll
            for (int j = 0; j < kTiles; ++j) *reinterpret_cast<float2*>(to + j * 8 + 2 * t4) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
            if (t4 == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m[h], all[h]);
          }
        }
      }
    }
  }
}

constexpr int kJoinThreads = 512;
// Finishes the heads that the runs' ends cut: some warps of a CTA per head and row, as many as there are warps
// for, lanes along the columns, pieces dealt to the warps and joined in a fixed order.  The lists are those
// of the step, written before the kernel ahead passed its own wait; the pieces are that kernel's.  Bound:
// latency (a round trip for eight pieces a warp): 1.5 us for 32 heads of 8 pieces, 5 us for 32 rows of 220.  A ticket
// per head in the kernel ahead, whose last piece's CTA did this, took 1.2 us a piece and 20 us for 71 rows of 18.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads)
kv_join_kernel(KvView V, T* out) {
  constexpr int kWarps = kJoinThreads / 32, kVecs = (D + 127) / 128;       // float4 of a lane
  __shared__ float4 fold[kWarps][kVecs * 32];
  __shared__ float2 stat[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = V.counts[KV_JOINS], slot_rows = V.slot_rows, units = n * slot_rows;
  int split = kWarps;                                // warps of a unit
  while (split > 1 && (long long)units * split > (long long)gridDim.x * kWarps) split /= 2;
  const int per_cta = kWarps / split, part = warp % split;
  bool waited = false;
  for (int u0 = blockIdx.x * per_cta; u0 < units; u0 += gridDim.x * per_cta) {
    const int u = u0 + warp / split;
    int4 join = make_int4(0, 0, 0, 0);
    int row = 0, pieces = 0, r = 0;
    if (u < units) {
      join = V.joins[u / slot_rows];                 // {first run, last run << 16; place; head << 16, row block; new tokens}
      r = u % slot_rows;
      row = (join.z & 0xffff) * V.rows_per_block + r;
      if (row < join.w * V.group) pieces = (join.x >> 16) - (join.x & 0xffff) + 1;
    }
    if (!waited) pdl_wait();
    waited = true;
    float m = -INFINITY, l = 0.f;
    float4 acc[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = part; p0 < pieces; p0 += 8 * split) {
      float2 st[8];
      float4 x[8][kVecs];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + e * split;
        st[e] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) x[e][v] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p < pieces) {                            // piece p: the first run's second slot, every other one's first
          const float* from = V.partials + (size_t)(2 * ((join.x & 0xffff) + p) + (p == 0)) * V.slot_floats + (size_t)r * (D + 4);
          st[e] = __ldcg(reinterpret_cast<const float2*>(from + D));
#pragma unroll
          for (int v = 0; v < kVecs; ++v)
            if (v * 32 + lane < D / 4) x[e][v] = __ldcg(reinterpret_cast<const float4*>(from) + v * 32 + lane);
        }
      }
      float top = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, st[e].x);
      const float base = top == -INFINITY ? 0.f : top, shrink = power(m - base);
      m = top;
      l *= shrink;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(acc[v].x * shrink, acc[v].y * shrink, acc[v].z * shrink, acc[v].w * shrink);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = power(st[e].x - base);
        l = fmaf(st[e].y, f, l);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          acc[v].x = fmaf(f, x[e][v].x, acc[v].x);
          acc[v].y = fmaf(f, x[e][v].y, acc[v].y);
          acc[v].z = fmaf(f, x[e][v].z, acc[v].z);
          acc[v].w = fmaf(f, x[e][v].w, acc[v].w);
        }
      }
    }
    if (split > 1) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) fold[warp][v * 32 + lane] = acc[v];
      if (lane == 0) stat[warp] = make_float2(m, l);
      __syncthreads();
      if (part == 0) {
        for (int k = 1; k < split; ++k) m = fmaxf(m, stat[warp + k].x);
        const float base = m == -INFINITY ? 0.f : m;
        l = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < split; ++k) {
          const float f = power(stat[warp + k].x - base);
          l = fmaf(stat[warp + k].y, f, l);
#pragma unroll
          for (int v = 0; v < kVecs; ++v) {
            const float4 x = fold[warp + k][v * 32 + lane];
            acc[v].x = fmaf(f, x.x, acc[v].x);
            acc[v].y = fmaf(f, x.y, acc[v].y);
            acc[v].z = fmaf(f, x.z, acc[v].z);
            acc[v].w = fmaf(f, x.w, acc[v].w);
          }
        }
      }
    }
    if (part == 0 && pieces > 0) {
      const int t = row / V.group;
      T* to = out + (((int64_t)join.y * V.max_new + t) * V.n_heads + (join.z >> 16) * V.group + row - t * V.group) * D;
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
        if (v * 32 + lane < D / 4)
          reinterpret_cast<uint2*>(to)[v * 32 + lane] =
              make_uint2(Num<T>::from2(acc[v].x / l, acc[v].y / l), Num<T>::from2(acc[v].z / l, acc[v].w / l));
    }
    if (split > 1) __syncthreads();
  }
  if (!waited) pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) V.counts[KV_TAKEN] = 0;
}

// What to do with the kernels for a type, head dimension and row tiles: few rows leave the tile's keys to more warps.
// Heads of 64 and 128 come here with up to 16 rows; more are the wide kernel's.
template <typename T, int D, int WR, int WK, typename F>
cudaError_t with(F f) {
  using S = Shape<D, WR, WK>;
  return f(kv_attention_kernel<T, D, WR, WK>, S::kThreads, S::kSmem);
}
template <typename T, int D, typename F>
cudaError_t with_rows(int row_tiles, F f) {
  if constexpr (D == 64 || D == 128) {
    return with<T, D, 1, 4>(f);
  } else if constexpr (D < 128) {
    if (row_tiles == 1) return with<T, D, 1, 4>(f);
    if (row_tiles == 2) return with<T, D, 2, 4>(f);
    if (row_tiles == 4) return with<T, D, 4, 2>(f);
    return with<T, D, 8, 1>(f);
  } else {                               // 128 registers of output: four warps that compute
    if (row_tiles == 1) return with<T, D, 1, 4>(f);
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
template <typename T>
cudaError_t launch_join(const lif_kv* kv, void* out, cudaStream_t st) {
  auto go = [&](auto kernel) { return launch_k2(kernel, dim3(kv->n_sm), dim3(kJoinThreads), 0, st, 1, 1, kv->v, (T*)out); };
  switch (kv->desc.head_dim) {
    case 64: return go(kv_join_kernel<T, 64>);
    case 80: return go(kv_join_kernel<T, 80>);
    case 96: return go(kv_join_kernel<T, 96>);
    case 128: return go(kv_join_kernel<T, 128>);
    default: return go(kv_join_kernel<T, 256>);
  }
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
// read once, up to what registers and shared memory take (128 rows, 64 at 256 columns).  The wide kernel's
// blocks are the 128 rows of a tensor-core tile however few are there.
int kv_row_tiles(const lif_kv_desc& d) {
  const int rows = d.n_heads / d.n_kv_heads * d.max_new, most = d.head_dim <= 128 ? 8 : 4;
  int t = 1;
  while (t < most && t * 16 < rows) t *= 2;
  return t > 1 && (d.head_dim == 64 || d.head_dim == 128) ? most : t;
}

bool kv_attention_configure(lif_kv* kv, int* ctas_per_sm) {
  if (!encode_map(&kv->maps.wide, kv->desc, 64, CU_TENSOR_MAP_SWIZZLE_128B)) return false;
  if (kv->desc.head_dim == 96 && !encode_map(&kv->maps.rest, kv->desc, 32, CU_TENSOR_MAP_SWIZZLE_64B)) return false;
  if (kv_is_wide(kv->desc)) return kv_wide_configure(kv, ctas_per_sm) == cudaSuccess;
  return with_kernel(kv, [&](auto kernel, int threads, int smem) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, kernel, threads, smem);
    return e;
  }) == cudaSuccess;
}

cudaError_t launch_kv_attention(const lif_kv* kv, int layer, const void* q, void* out, cudaStream_t st) {
  const lif_kv_desc& d = kv->desc;
  AttendArgs a;
  a.q = q;
  a.out = out;
  a.scale_log2 = kv->scale * 1.4426950408889634f;
  a.layer = layer;
  a.pages = (const char*)d.dev_pages + (size_t)layer * d.n_pages * kv_page_elems(d) * 2;
  cudaError_t e = kv_is_wide(d) ? launch_kv_attention_wide(kv, a, st) : with_kernel(kv, [&](auto kernel, int threads, int smem) {
    return launch_k2(kernel, dim3(kv->v.ctas), dim3(threads), smem, st, 1, 1, kv->maps, kv->v, a);
  });
  if (e != cudaSuccess) return e;
  return d.dtype == LIF_TYPE_F16 ? launch_join<__half>(kv, out, st) : launch_join<__nv_bfloat16>(kv, out, st);
}

}  // namespace lif
