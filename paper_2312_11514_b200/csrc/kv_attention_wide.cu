// Attention over the paged cache where more than 16 rows share a key-value head (a long step, many query heads
// over few), head dimensions 64 and 128: the formula, the split into runs and the join are kv_attention.cu's.
//
// Why another kernel.  One row block of 128 is a tile of the tcgen05 tensor cores, where mma.sync took eight
// times as long and was the bound: 64 new tokens of 4 sequences of 8000, 32 heads over 8, 125 us there and 69 here
// (two row blocks read keys and values each: 262 MB, 58% of measured HBM); 4 tokens of
// 64 heads over 8, 16 sequences of 4000, 85 and 66; 71 heads over one of 64, 8 sequences of 60000, 65 and 39.  Only the
// shortest lose: 71 heads, 8 sequences of 1500 .. 32000, 16.1 and 17.0 (lengths are known on the device alone).  What
// is left is one exponential per row and key (16 a clock and SM): with 128 rows a tile of 64 keys takes 512 clocks of
// those, two thirds of what its bytes take HBM for D = 128.  Few rows leave lanes of the softmax idle but cost no more.
// A CTA is two halves of six warps that share nothing but the allocation of tensor memory, so that one's tensor
// cores and copies run beside the other's exponentials.  (Two CTAs an SM would do the same, but the allocation waits
// without a limit where CTAs compete for it; one CTA takes all 512 columns at once.)  In a half:
//
//   warp 5      issues the products, S = Q K^T of tile i ahead of O += P V of tile i - 1
//   warp 4      moves keys and values (separate rings, since keys are done with a softmax earlier), and the
//               rows of queries when a head begins
//   warps 0-3   a thread per row: its 64 scores from tensor memory, weights back into the same columns as the
//               second product's operand, no exchange between threads; the output at the end of a head
//
// Tensor memory, 256 columns a half: scores of two tiles, 64 columns each, whose first 32 then hold the weights; the
// output, D columns.  It is rescaled in place when a row's reference moves (kSlack), which few tiles ask for.
//
// Keys that rows differ about: scores are replaced by -inf, values that no row sees are cleared in shared memory,
// and where a value is not finite that some rows see and others do not, the tile's second product is formed
// one by one outside the tensor cores (0 times infinity is not 0).
//
// Precision as in kv_attention.cu, but for the sum of a row's weights, which is that of the weights before
// their rounding (the exponentials and these sums are the bound here): each weight's rounding then stands in the
// output as it does in the weights.
#include "kv_attention.cuh"

namespace lif {
namespace {

constexpr int kWideRows = 128, kHalfThreads = 192, kWideThreads = 2 * kHalfThreads, kInfos = 8;
constexpr int kScoreColumns = kKvTile, kOutColumn = 2 * kKvTile, kColumns = 256;   // of tensor memory, a half

constexpr int kMaxStages = 4;
template <int D>
struct Wide {
  static constexpr int kTileBytes = kKvTile * D * 2;                     // keys, or values
  // The tile of queries has 128 rows for the tensor cores; memory is laid out for those that can be there, and
  // rows behind them are whatever the ring holds there (a row's scores are its own).  What that saves are more stages.
  static constexpr int kRoom = (227 * 1024 / 2 - 1024) / 1024 * 1024;    // of a half, beside its state
  static int rows(int slot_rows) { return slot_rows <= 32 ? 32 : slot_rows <= 64 ? 64 : kWideRows; }
  static int stages(int slot_rows) {
    const int n = (kRoom - rows(slot_rows) * D * 2) / (2 * kTileBytes);
    return n > kMaxStages ? kMaxStages : n;
  }
  static constexpr int kHalfBytes = kRoom + 1024, kSmem = 2 * kHalfBytes;
  static_assert(kRoom - kWideRows * D * 2 >= 4 * kTileBytes && kInfos >= kMaxStages + 3 && kOutColumn + D <= kColumns, "");
};
struct WideShape {
  int rows, stages;                // of queries; of keys, and of values
};

struct __align__(16) WideState {
  StageInfo info[kInfos];
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
  uint64_t q_full, q_empty;        // rows of queries: here; read by the last product that needs them
  uint64_t s_full[2], p_full[2];   // scores; weights (and cleared values)
  uint64_t o_done, o_empty;        // a tile's second product; the output, read
  uint64_t drained;
  int by_hand[2];                  // the second product is not the tensor cores'
  uint32_t columns;                // (the first half's)
};
static_assert(sizeof(WideState) <= 1024, "");

// ---- tensor cores ------------------------------------------------------------------------------------

// Shared-memory operand in rows of 128 bytes, permuted as the 128-byte swizzle does it.  `across`: bytes between
// 64-element columns of an operand whose rows are the reduction (values); eight rows lie 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t across) {
  return (uint64_t)((at >> 4) & 0x3fff) | (uint64_t)(across >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 sums of 128 x n; the second operand's rows along its columns (keys) or along the reduction (values)
template <typename T>
__device__ __forceinline__ constexpr uint32_t product(int n, bool along) {
  constexpr uint32_t type = sizeof(T) == 2 && Num<T>::kExponent == 0x7f807f80u ? 1u : 0u;   // bf16 : f16
  return 1u << 4 | type << 7 | type << 10 | (along ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kWideRows >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t how, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
// the barrier is told when all products issued so far are done
__device__ __forceinline__ void products_done(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tensor_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of the thread's row
__device__ __forceinline__ void columns_load(uint32_t* r, uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at) : "memory");
}
__device__ __forceinline__ void columns_here() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void columns_store(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void columns_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ bool elect() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
// (bounded; the warp's lanes go on, or give up, together)
__device__ __forceinline__ bool warp_wait(uint64_t* bar, unsigned parity) { return __all_sync(~0u, mbar_wait(bar, parity)); }

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}

// ---- the loading warp -----------------------------------------------------------------------------------

template <typename T, int D>
__device__ __forceinline__ bool wide_feed(const KvMaps& maps, const KvView& V, const AttendArgs& a, uint32_t keys, uint32_t values,
                                          unsigned char* queries, WideState* st, WideShape shape, int who, int4 plan, int4 step) {
  using S = Wide<D>;
  constexpr int kChunks = D / 64;
  const int lane = threadIdx.x & 31;
  const int page_tokens = 1 << V.page_shift, box = min(page_tokens, kKvTile);
  Walk walk(V, who, plan, step);
  const Cursor& at = walk.at;
  int k_stage = 0, v_stage = 0, piece = 0;
  unsigned k_turn = 0, v_turn = 0;
  bool ok = true;
  // a lane's box: chunk and page of the tile (at most 8 pages of 2 chunks); the values' one is issued a tile later
  int page = 0, row = 0, head = 0, n_pages = 0, i = 0, issued_v = 0;
  auto values_of = [&]() {
    if (!__all_sync(~0u, mbar_wait(st->v_empty + v_stage, v_turn ^ 1))) return false;
    if (lane == 0) mbar_expect_tx(st->v_full + v_stage, n_pages * box * D * 2);
    __syncwarp();
    const int p = lane / kChunks, chunk = lane % kChunks;
    if (p < n_pages)
      tensor_g2s(values + v_stage * S::kTileBytes + chunk * 8192 + p * box * 128, &maps.wide, chunk * 64, row, V.n_kv_heads + head,
                 page, a.layer, st->v_full + v_stage);
    if (++v_stage == shape.stages) v_stage = 0, v_turn ^= 1;
    ++issued_v;
    return true;
  };
  for (; ok && !walk.last; ++i) {
    walk.begin(V, lane);
    if (!__all_sync(~0u, mbar_wait(st->k_empty + k_stage, k_turn ^ 1))) {
      ok = false;
      break;
    }
    const int p = lane / kChunks, chunk = lane % kChunks;
    const int next_page = __shfl_sync(~0u, walk.held, walk.j0 - walk.held_from + p & 31);
    const int next_row = walk.k0 & (page_tokens - 1), next_n = walk.n_pages, next_head = at.head;
    if (lane == 0) {
      st->info[i % kInfos] = walk.info(V);
      mbar_expect_tx(st->k_full + k_stage, next_n * box * D * 2);
    }
    __syncwarp();
    if (p < next_n)
      tensor_g2s(keys + k_stage * S::kTileBytes + chunk * 8192 + p * box * 128, &maps.wide, chunk * 64, next_row, next_head, next_page,
                 a.layer, st->k_full + k_stage);
    if (++k_stage == shape.stages) k_stage = 0, k_turn ^= 1;
    // the values of the tile before
    if (i > 0 && !values_of()) {
      ++i;
      ok = false;
      break;
    }
    page = next_page;
    row = next_row;
    n_pages = next_n;
    head = next_head;
    if (walk.opens) {
      if (!__all_sync(~0u, mbar_wait(&st->q_empty, (piece & 1) ^ 1))) {
        ++i;
        ok = false;
        break;
      }
      const int row0 = at.block * kWideRows, rows = min(kWideRows, at.news * V.group - row0);
      // lanes along a row's 16-byte pieces: [64 columns][row][128 bytes], permuted as the keys are; row r is head
      // (row0 + r) % group of token (row0 + r) / group
      constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces;
      const int c = lane % kPieces;
      int r = lane / kPieces, t = (row0 + r) / V.group, h = row0 + r - t * V.group;
      const T* src = reinterpret_cast<const T*>(a.q) + (((int64_t)at.b * V.max_new + t) * V.n_heads + at.head * V.group + h) * D + 8 * c;
      const int64_t next_token = (int64_t)(V.n_heads - V.group) * D;
      unsigned char* to = queries + (c / 8) * shape.rows * 128 + r * 128;
#pragma unroll 4
      for (; r < rows; r += kAtOnce, to += kAtOnce * 128) {
        copy_async16(to + ((c & 7) ^ (r & 7)) * 16, src);
        src += kAtOnce * D;
        for (h += kAtOnce; h >= V.group; h -= V.group) src += next_token;
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&st->q_full)) : "memory");
      ++piece;
    }
    walk.advance(V);
  }
  if (ok) ok = values_of();
  // nobody leaves while copies are on their way
  for (int k = 0; k < min(i, shape.stages); ++k) {
    if (k_stage == 0) k_turn ^= 1;
    k_stage = k_stage == 0 ? shape.stages - 1 : k_stage - 1;
    mbar_wait(st->k_full + k_stage, k_turn);
  }
  for (int k = 0; k < min(issued_v, shape.stages); ++k) {
    if (v_stage == 0) v_turn ^= 1;
    v_stage = v_stage == 0 ? shape.stages - 1 : v_stage - 1;
    mbar_wait(st->v_full + v_stage, v_turn);
  }
  own_copies_wait();
  return ok;
}

// ---- the warp that issues the products ------------------------------------------------------------------------
// All its lanes walk and wait, one issues: what it computes is the warp's and stays in uniform registers, which is
// where the tensor cores' instructions take their operands from (one lane alone: 2000 clocks a tile, so: 900).

template <typename T, int D>
__device__ __forceinline__ bool wide_products(uint32_t keys, uint32_t values, uint32_t queries, WideState* st, WideShape shape, uint32_t columns) {
  using S = Wide<D>;
  const uint64_t q0 = operand(queries, 16), k0 = operand(keys, 16), v0 = operand(values, 8192);
  int k_stage = 0, v_stage = 0, piece_s = 0, piece_o = 0, flags_before = 0;
  unsigned k_turn = 0, v_turn = 0;
  bool add = false;
  auto second = [&](int j, int flags) {              // O += P V of tile j
    if (!warp_wait(st->v_full + v_stage, v_turn)) return false;
    if (flags & kOpens) {
      if (!warp_wait(&st->o_empty, (piece_o & 1) ^ 1)) return false;
      ++piece_o;
      add = false;
    }
    if (!warp_wait(st->p_full + (j & 1), j >> 1 & 1)) return false;
    tensor_after();
    const bool by_hand = __shfl_sync(~0u, st->by_hand[j & 1], 0) != 0;
    if (elect()) {
      if (by_hand) {
        mbar_arrive(st->v_empty + v_stage);
        mbar_arrive(&st->o_done);
      } else {
        const uint64_t v = v0 + v_stage * (S::kTileBytes >> 4);
        const uint32_t weights = columns + (j & 1) * kScoreColumns;
        mma_ts(columns + kOutColumn, weights, v, product<T>(D, true), add);
#pragma unroll
        for (int k = 1; k < kKvTile / 16; ++k)
          mma_ts(columns + kOutColumn, weights + k * 8, v + k * (2048 >> 4), product<T>(D, true), true);
        products_done(&st->o_done);
        products_done(st->v_empty + v_stage);
      }
    }
    __syncwarp();
    add = true;
    if (++v_stage == shape.stages) v_stage = 0, v_turn ^= 1;
    return true;
  };
  for (int i = 0;; ++i) {
    if (!warp_wait(st->k_full + k_stage, k_turn)) return false;
    const int flags = __shfl_sync(~0u, st->info[i % kInfos].flags, 0);
    if (flags & kOpens) {
      if (!warp_wait(&st->q_full, piece_s++ & 1)) return false;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the queries' copies are not the tensor cores' kind
    }
    tensor_after();
    if (elect()) {
      const uint64_t k = k0 + k_stage * (S::kTileBytes >> 4);
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
        mma_ss(columns + (i & 1) * kScoreColumns, q0 + (e / 4) * (shape.rows * 128 >> 4) + ((e % 4) * 32 >> 4),
               k + ((e / 4) * 8192 + (e % 4) * 32 >> 4), product<T>(kKvTile, false), e > 0);
      products_done(st->s_full + (i & 1));
      products_done(st->k_empty + k_stage);
      if (flags & kCloses) products_done(&st->q_empty);
    }
    __syncwarp();
    if (++k_stage == shape.stages) k_stage = 0, k_turn ^= 1;
    if (i > 0 && !second(i - 1, flags_before)) return false;
    flags_before = flags;
    if (flags & kLast) return second(i, flags);
  }
}

// ---- a thread per row -------------------------------------------------------------------------------------

template <typename T, int D>
__device__ __forceinline__ bool wide_rows(const KvView& V, const AttendArgs& a, unsigned char* values, WideState* st,
                                          WideShape shape, uint32_t columns, int warp) {
  using S = Wide<D>;
  const int lane = threadIdx.x & 31, r = warp * 32 + lane;
  const uint32_t mine = columns + ((uint32_t)(warp * 32) << 16);
  const uint32_t out_at = mine + kOutColumn;
  float m = -INFINITY, sum = 0.f;
  int upto = 0, rows = 0, v_stage = 0;
  unsigned v_turn = 0;
  bool starts = false, idle = false;
  const int reach = V.window > 0 ? V.window : 0x7fffffff;
  // A barrier tells a phase from its neighbours only.  So every warp, with rows or without, sees the second product
  // of every tile done before it hands over the next tile's weights (which that product could not follow otherwise):
  // no phase begins that it has not seen the one before the last of.  It is done by then, as a rule.
  int done = 0;
  auto done_through = [&](int tile) {
    for (; done <= tile; ++done)
      if (!warp_wait(&st->o_done, done & 1)) return false;
    return true;
  };
#pragma unroll 1
  for (int i = 0;; ++i) {
    const int half = i & 1;
    if (!warp_wait(st->s_full + half, i >> 1 & 1) ) return false;
    tensor_after();
    const StageInfo at = st->info[i % kInfos];
    const bool opens = at.flags & kOpens;
    if (opens) {
      starts = at.flags & kStarts;
      rows = min(kWideRows, at.news * V.group - at.row0);
      idle = warp * 32 >= rows;
      upto = at.tokens - at.news + min((at.row0 + r) / V.group, at.news - 1);
      m = -INFINITY;
      sum = 0.f;
    }
    const uint32_t scores = mine + half * kScoreColumns;
    bool one_by_one = false, clear = false;
    unsigned char* v = values + v_stage * S::kTileBytes;
    if (at.flags & kEdge) {
      const Edge edge(V, at);
      clear = edge.clear(at, at.k0, kKvTile);
      const bool differ = edge.differ(at, at.k0, kKvTile);
      if (clear || differ) {
        if (!warp_wait(st->v_full + v_stage, v_turn)) return false;
        // every warp looks at all that rows differ about (so all of them find the same), and clears a quarter
        constexpr int kPieces = D / 8;
        const int c = lane % kPieces;
        bool odd = false;
        for (int k = lane / kPieces; k < kKvTile; k += 32 / kPieces) {
          uint4* p = reinterpret_cast<uint4*>(v + piece<D>(k, c));
          if (!edge.none(at, at.k0 + k)) odd = odd || (differ && any_not_finite<T>(*p));
          else if (k >> 4 == warp) *p = make_uint4(0, 0, 0, 0);
        }
        one_by_one = __any_sync(~0u, odd);
        if (clear) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor cores, later copies
      }
    }
    if (!idle) {
      uint32_t x[64];
      columns_load(x, scores);
      columns_load(x + 32, scores + 32);
      columns_here();
      float* s = reinterpret_cast<float*>(x);
      if (at.flags & kEdge) {
#pragma unroll
        for (int c = 0; c < 64; ++c) {
          const int key = at.k0 + c;
          if (key > upto || upto - key >= reach) s[c] = -INFINITY;
        }
      }
      float top4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int c = 4; c < 64; ++c) top4[c & 3] = fmaxf(top4[c & 3], s[c]);
      const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
      const bool above = too_far<T>(top, a.scale_log2, m);
      if (__any_sync(~0u, above)) {                  // (each row by itself: rows that are not there hold anything)
        const float now = above ? new_reference<T>(top, a.scale_log2) : m;
        const float shrink = power(m - (now == -INFINITY ? 0.f : now));
        m = now;
        sum *= shrink;
        if (!opens) {
          if (!done_through(i - 1)) return false;
          tensor_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            columns_load(o, out_at + c);
            columns_here();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
            columns_store(out_at + c, o);
          }
          columns_stored();
        }
      }
      const float base = m == -INFINITY ? 0.f : m;
      uint32_t w[32];
      float2 add[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      const float2 factor = make_float2(a.scale_log2, a.scale_log2), offset = make_float2(-base, -base);
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        const float2 e = fma2(make_float2(s[2 * c], s[2 * c + 1]), factor, offset);
        const float2 p = make_float2(power(e.x), power(e.y));
        w[c] = Num<T>::from2(p.x, p.y);
        add[c & 1] = add2(add[c & 1], p);
      }
      sum += (add[0].x + add[0].y) + (add[1].x + add[1].y);
      if (!one_by_one) {
        columns_store(scores, w);
      } else {
        // the products outside the tensor cores, in the output where it lies (which begins here if the head does)
        if (!opens && !done_through(i - 1)) return false;
        tensor_after();
        uint32_t kept[32];                           // (in local memory: this path is rare)
        for (int c = 0; c < 32; ++c) kept[c] = w[c];
        const volatile uint32_t* weights = kept;
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          uint32_t o[32];
          if (!opens) {
            columns_load(o, out_at + c0);
            columns_here();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0;
          }
#pragma unroll 1
          for (int k = 0; k < kKvTile; ++k) {
            if (at.k0 + k > upto || upto - (at.k0 + k) >= reach) continue;
            const float2 pair = Num<T>::to2(weights[k >> 1]);
            const float weight = k & 1 ? pair.y : pair.x;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint4 bits = *reinterpret_cast<const uint4*>(v + piece<D>(k, c0 / 8 + q));
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 y = Num<T>::to2((&bits.x)[e]);
                o[8 * q + 2 * e] = __float_as_uint(fmaf(weight, y.x, __uint_as_float(o[8 * q + 2 * e])));
                o[8 * q + 2 * e + 1] = __float_as_uint(fmaf(weight, y.y, __uint_as_float(o[8 * q + 2 * e + 1])));
              }
            }
          }
          __syncwarp();
          columns_store(out_at + c0, o);
        }
      }
      columns_stored();
    }
    if (!done_through(i - 1)) return false;
    if (r == 0) st->by_hand[half] = one_by_one;
    tensor_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(st->p_full + half);
    if (++v_stage == shape.stages) v_stage = 0, v_turn ^= 1;

    if (at.flags & kCloses) {
      if (!done_through(i)) return false;
      tensor_after();
      if (!idle) {
        const bool whole = starts && (at.flags & kEnds);
        T* out = reinterpret_cast<T*>(a.out) + row_offset(V, at, r);
        // a piece that began before this run, or one that goes on behind it
        float* part = V.partials + (size_t)(2 * at.run + starts) * V.slot_floats + (size_t)r * (D + 4);
        const float inv = 1.f / sum;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          columns_load(o, out_at + c);
          columns_here();
          const float* f = reinterpret_cast<const float*>(o);
          if (r < rows && whole) {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(out + c + e) =
                  make_uint4(Num<T>::from2(f[e] * inv, f[e + 1] * inv), Num<T>::from2(f[e + 2] * inv, f[e + 3] * inv),
                             Num<T>::from2(f[e + 4] * inv, f[e + 5] * inv), Num<T>::from2(f[e + 6] * inv, f[e + 7] * inv));
          } else if (r < rows) {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(part + c + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
          }
          __syncwarp();
        }
        if (!whole && r < rows) *reinterpret_cast<float2*>(part + D) = make_float2(m, sum);
      }
      tensor_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&st->o_empty);
      if (at.flags & kLast) return true;
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kWideThreads, 1)
kv_attention_wide_kernel(const __grid_constant__ KvMaps maps, KvView V, AttendArgs a, WideShape shape) {
  using S = Wide<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  // A warp reaches the tensor memory lanes of its number modulo 4, so rows are warps 0-3 of one half and 8-11 of
  // the other; 4-7 load and issue.
  const int number = __shfl_sync(~0u, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int half = number >= 6, role = number < 4 ? 0 : number >= 8 ? 0 : number % 2 == 0 ? 4 : 5;
  unsigned char *queries = smem + half * S::kHalfBytes, *keys = queries + shape.rows * D * 2,
                *values = keys + shape.stages * S::kTileBytes;
  WideState* st = reinterpret_cast<WideState*>(queries + S::kRoom);
  WideState* first = reinterpret_cast<WideState*>(reinterpret_cast<unsigned char*>(st) - half * S::kHalfBytes);
  if (role == 4 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.wide) : "memory");
    for (int i = 0; i < shape.stages; ++i) {
      mbar_init(st->k_full + i, 1);
      mbar_init(st->k_empty + i, 1);
      mbar_init(st->v_full + i, 1);
      mbar_init(st->v_empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(st->s_full + i, 1);
      mbar_init(st->p_full + i, 4);
    }
    mbar_init(&st->q_full, 32);
    mbar_init(&st->q_empty, 1);
    mbar_init(&st->o_done, 1);
    mbar_init(&st->o_empty, 4);
    mbar_init(&st->drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  const int4 step = *reinterpret_cast<const int4*>(V.counts + KV_TILES);
  // halves are numbered so that few shares go to as many SMs
  const int who = half * gridDim.x + blockIdx.x;
  const int4 plan = V.run_plan[who];
  if ((int)blockIdx.x >= step.y) return;             // (the whole CTA, before it holds anything)
  if (number == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&st->columns)), "n"(2 * kColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tensor_before();
  __syncthreads();
  tensor_after();
  const uint32_t all = __shfl_sync(~0u, first->columns, 0), columns = all + half * kColumns;
  if (who < step.y) {
    bool ok = true;
    if (role == 4) {
      ok = wide_feed<T, D>(maps, V, a, smem_u32(keys), smem_u32(values), queries, st, shape, who, plan, step);
    } else if (role == 5) {
      ok = wide_products<T, D>(smem_u32(keys), smem_u32(values), smem_u32(queries), st, shape, columns);
      if (elect()) products_done(&st->drained);      // none is under way when the columns are given back
      warp_wait(&st->drained, 0);
    } else {
      ok = wide_rows<T, D>(V, a, values, st, shape, columns, number % 4);
    }
    if (!ok) flag_timeout(V.counts + LIF_KV_CNT_STATUS);
  }
  tensor_before();
  __syncthreads();
  tensor_after();
  if (number == 5)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(all), "n"(2 * kColumns) : "memory");
}

template <int D, typename T, typename F>
cudaError_t with(const lif_kv* kv, F f) {
  using S = Wide<D>;
  return f(kv_attention_wide_kernel<T, D>, S::kSmem, WideShape{S::rows(kv->v.slot_rows), S::stages(kv->v.slot_rows)});
}
template <typename F>
cudaError_t with_wide(const lif_kv* kv, F f) {
  const bool half = kv->desc.dtype == LIF_TYPE_F16;
  if (kv->desc.head_dim == 64) return half ? with<64, __half>(kv, f) : with<64, __nv_bfloat16>(kv, f);
  return half ? with<128, __half>(kv, f) : with<128, __nv_bfloat16>(kv, f);
}

}  // namespace

cudaError_t kv_wide_configure(const lif_kv* kv, int* ctas_per_sm) {
  return with_wide(kv, [&](auto kernel, int smem, WideShape) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, kernel, kWideThreads, smem);
    if (e == cudaSuccess && *ctas_per_sm > 0) *ctas_per_sm = 2;          // two halves
    return e;
  });
}

cudaError_t launch_kv_attention_wide(const lif_kv* kv, const AttendArgs& a, cudaStream_t st) {
  return with_wide(kv, [&](auto kernel, int smem, WideShape shape) {
    return launch_k2(kernel, dim3(kv->v.ctas / 2), dim3(kWideThreads), smem, st, 1, 1, kv->maps, kv->v, a, shape);
  });
}

}  // namespace lif
