// Attention of a step's new tokens over the paged key-value cache.
//
//   out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale <q_row, k_j> - max_j)
//
// Rows: the new tokens' query heads that share a key-value head, `group` x tokens of them (1 .. 16
// mostly), in blocks of 16 x MT.  Every key and value is read once per row block; bound: HBM, until
// rows x heads make the tensor cores or the exponentials one (a single key-value head under many query heads).
//
// Split.  The step's work is numbered in tiles of 64 keys (kv_plan) and every CTA takes an equal run
// of them, across heads and sequences, so that one long sequence, many short ones and anything ragged
// between fill the chip alike.  A head that a run's end cuts is finished by kv_join_kernel from the
// pieces' {max, sum, unnormalised output}, in a fixed order.
//
// Tile.  64 keys and values come through a ring of shared-memory stages by 16-byte asynchronous
// copies: the rows of a tile belong to pages of any size, rows past the end are filled with zeros
// instead of read, and the 16-byte pieces of a row are stored in the permuted order that makes
// ldmatrix free of bank conflicts.  The ring runs on across heads and sequences; queries travel with
// the first tile of their head.  Of a tile each of the 8 warps multiplies 8 keys by all rows
// (mma m16n8k16, rows = M), the maxima are exchanged through shared memory, the weights go there in
// 16 bits, and each warp then multiplies all 64 weights by its share of the value columns: no key,
// value or output element is held twice, and no warp's sums need to be joined with another's.
//
// Precision.  Scores, maxima, sums and outputs are fp32.  Weights are rounded to the cache's type
// for the second product (at most half a unit in the last place of each, like the rounding of the
// output); the sum is that of the rounded weights, so that they add up to one exactly as they are used.
#include "kv_internal.cuh"

namespace lif {
namespace {

constexpr int kWarps = kThreads / 32;

struct AttendArgs {
  const void *q, *pages;       // pages: this layer's
  void* out;
  float scale_log2;            // scale * log2(e): weights are powers of two
};

__device__ __forceinline__ void copy_async16_or_zero(uint32_t smem, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldm_x4(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm_x2(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(at) : "memory");
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

// Where 16-byte piece c of row r lies in a tile of rows of D elements: any 8 consecutive rows' pieces
// c fall into different banks.
template <int D>
__device__ __forceinline__ int piece(int r, int c) {
  if (D % 64 == 0) return r * (D / 8) + (c ^ (r & 7));
  if (D == 80) return r * 10 + (c ^ (r >> 2 & 1));       // rows 160 bytes apart: r and r + 4 meet
  return r * 12 + (c ^ (r >> 1 & 3));                    // D = 96, rows 192 bytes apart: every other one
}

template <int D, int MT>
struct Shape {
  static constexpr int kRows = 16 * MT;
  static constexpr int kTileBytes = kKvTile * D * 2;                     // keys, or values
  static constexpr int kQueryBytes = kRows * D * 2;
  static constexpr int kStage = 2 * kTileBytes + kQueryBytes;
  static constexpr int kFixed = kRows * kKvTile * 2 + kRows * kWarps * 4;  // weights, maxima
  // Two CTAs an SM where three stages fit twice: one computes while the other waits.
  static constexpr int kTwo = (113 * 1024 - kFixed) / kStage, kOne = (226 * 1024 - kFixed) / kStage;
  static constexpr int kCtas = kTwo >= 3 ? 2 : 1;
  static constexpr int kWanted = kCtas == 2 ? kTwo : kOne;
  static constexpr int kStages = kWanted > 6 ? 6 : kWanted;
  static constexpr int kSmem = kStages * kStage + kFixed;
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

template <typename T, int D, int MT>
__global__ void __launch_bounds__(kThreads, Shape<D, MT>::kCtas)
kv_attention_kernel(KvView V, AttendArgs a) {
  using S = Shape<D, MT>;
  constexpr int kPieces = D / 8;                     // 16-byte pieces of a row
  constexpr int kSteps = D / 16;                     // k steps of the first product
  constexpr int kCols = (kPieces + kWarps - 1) / kWarps;   // 8-column tiles of a warp's share of the output
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t ring = smem_u32(smem), queries = ring + S::kStages * 2 * S::kTileBytes,
                 weights = queries + S::kStages * S::kQueryBytes;
  float* maxima = reinterpret_cast<float*>(smem + S::kSmem - S::kRows * kWarps * 4);   // [rows][warps]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;

  pdl_wait();
  pdl_trigger();      // the join may become resident; it waits for this kernel's end itself
  const int total = V.counts[KV_TILES], per_cta = V.counts[KV_TILES_PER_CTA];
  const int g0 = blockIdx.x * per_cta;
  if (g0 >= total) return;
  const int n_tiles = min(total - g0, per_cta);
  Cursor load;
  {
    const int4 p = V.cta_plan[blockIdx.x];
    load.enter(V, p.x, p.z, p.w);
    const int in = g0 - p.y, item = in / load.tiles;
    load.tile = in - item * load.tiles;
    load.head = item / load.blocks;
    load.block = item - load.head * load.blocks;
  }
  Cursor cur = load;
  const int64_t head_elems = (int64_t)D << V.page_shift, page_elems = head_elems * V.n_kv_heads * 2;
  const T* pages = reinterpret_cast<const T*>(a.pages);
  const T* q = reinterpret_cast<const T*>(a.q);

  int load_stage = 0, load_slot = -1;
  auto issue = [&](bool first) {
    const int k0 = (load.first_tile + load.tile) * kKvTile;
    const int lowest = kv_first_key(load.tokens, load.news, V.window);
    const int32_t* row_pages = V.table + (size_t)load.b * V.max_pages;
    const T* head = pages + load.head * head_elems;
    const uint32_t at = ring + load_stage * 2 * S::kTileBytes;
#pragma unroll
    for (int i = 0; i < (kKvTile * kPieces + kThreads - 1) / kThreads; ++i) {
      const int x = tid + i * kThreads, r = x / kPieces, c = x - r * kPieces;
      if ((kKvTile * kPieces) % kThreads == 0 || x < kKvTile * kPieces) {
        const int key = k0 + r;
        // a key that no row sees is not read, whatever it holds
        const bool seen = key < load.tokens && key >= lowest;
        const T* src = head;
        if (seen)
          src += row_pages[key >> V.page_shift] * page_elems + (key & ((1 << V.page_shift) - 1)) * D + 8 * c;
        const uint32_t to = at + piece<D>(r, c) * 16;
        copy_async16_or_zero(to, src, seen);
        copy_async16_or_zero(to + S::kTileBytes, src + (seen ? head_elems * V.n_kv_heads : 0), seen);
      }
    }
    if (first || load.tile == 0) {
      load_slot = load_slot + 1 == S::kStages ? 0 : load_slot + 1;
      const int row0 = load.block * S::kRows, rows = load.news * V.group - row0;
      const int rows16 = min(S::kRows, (rows + 15) & ~15);
      for (int x = tid; x < rows16 * kPieces; x += kThreads) {
        const int r = x / kPieces, c = x - r * kPieces;
        const int t = (row0 + r) / V.group, i = row0 + r - t * V.group;
        const bool real = r < rows;
        const T* src = q + (real ? (((int64_t)load.b * V.max_new + t) * V.n_heads + load.head * V.group + i) * D + 8 * c : 0);
        copy_async16_or_zero(queries + load_slot * S::kQueryBytes + piece<D>(r, c) * 16, src, real);
      }
    }
    load_stage = load_stage + 1 == S::kStages ? 0 : load_stage + 1;
    load.step(V);
  };

#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) {
    if (i < n_tiles) issue(i == 0);
    copies_commit();
  }

  float o[MT][kCols][4];               // rows g, g + 8 of every row tile; the warp's columns
  float m[MT][2], sum[MT][2];          // running maximum; this lane's share of the sum
  int upto[MT][2];                     // last key that the row sees
  uint32_t qf[MT == 1 ? kSteps : 1][4];
  int stage = 0, slot = -1, row_tiles = 0, piece_start = 0;
  for (int i = 0; i < n_tiles; ++i) {
    copies_wait<S::kStages - 2>();
    __syncthreads();                   // the tile is here; everybody is done with the last one
    if (i + S::kStages - 1 < n_tiles) issue(false);
    copies_commit();

    if (i == 0 || cur.tile == 0) {     // another head's rows
      slot = slot + 1 == S::kStages ? 0 : slot + 1;
      piece_start = cur.tile;
      const int row0 = cur.block * S::kRows, rows = cur.news * V.group - row0;
      row_tiles = min(MT, (rows + 15) / 16);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = (row0 + mt * 16 + g + 8 * h) / V.group;
          upto[mt][h] = cur.tokens - cur.news + min(t, cur.news - 1);
          m[mt][h] = -INFINITY;
          sum[mt][h] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[mt][j][e] = 0.f;
      }
      if (MT == 1) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
          ldm_x4(qf[k], queries + slot * S::kQueryBytes + piece<D>(lane & 15, 2 * k + (lane >> 4)) * 16);
      }
    }
    const uint32_t keys = ring + stage * 2 * S::kTileBytes, values = keys + S::kTileBytes;

    // scores of the warp's 8 keys
    float s[MT][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) s[mt][0] = s[mt][1] = s[mt][2] = s[mt][3] = 0.f;
#pragma unroll
    for (int k = 0; k < kSteps; k += 2) {
      uint32_t kf[4];
      const int r = warp * 8 + (lane & 7);
      if (k + 1 < kSteps) ldm_x4(kf, keys + piece<D>(r, 2 * k + (lane >> 3)) * 16);
      else ldm_x2(kf, keys + piece<D>(r, 2 * k + (lane >> 3 & 1)) * 16);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if (k + kk < kSteps) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            if (MT == 1) {
              mma(T(), s[0], qf[MT == 1 ? k + kk : 0], kf[2 * kk], kf[2 * kk + 1]);
            } else if (mt < row_tiles) {
              uint32_t qa[4];
              ldm_x4(qa, queries + slot * S::kQueryBytes + piece<D>(mt * 16 + (lane & 15), 2 * (k + kk) + (lane >> 4)) * 16);
              mma(T(), s[mt], qa, kf[2 * kk], kf[2 * kk + 1]);
            }
          }
        }
      }
    }
    const int k0 = (cur.first_tile + cur.tile) * kKvTile;
    const bool edge = k0 + kKvTile > cur.tokens - cur.news + 1 || (V.window > 0 && k0 <= cur.tokens - 1 - V.window);
    const int reach = V.window > 0 ? V.window : 0x7fffffff;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (MT > 1 && mt >= row_tiles) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[mt][e] *= a.scale_log2;
      if (edge) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = k0 + warp * 8 + 2 * t4 + (e & 1), last = upto[mt][e >> 1];
          if (key > last || last - key >= reach) s[mt][e] = -INFINITY;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = fmaxf(s[mt][2 * h], s[mt][2 * h + 1]);
        x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
        x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
        if (t4 == 0) maxima[(mt * 16 + g + 8 * h) * kWarps + warp] = x;
      }
    }
    __syncthreads();
    // weights 2^(s - max); a row that has seen nothing yet keeps max = -inf and weights 0
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (MT > 1 && mt >= row_tiles) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = mt * 16 + g + 8 * h;
        const float4 x = *reinterpret_cast<const float4*>(maxima + r * kWarps);
        const float4 y = *reinterpret_cast<const float4*>(maxima + r * kWarps + 4);
        const float top = fmaxf(fmaxf(fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)), fmaxf(fmaxf(y.x, y.y), fmaxf(y.z, y.w))), m[mt][h]);
        const float base = top == -INFINITY ? 0.f : top;
        const float shrink = exp2f(m[mt][h] - base);
        m[mt][h] = top;
        const uint32_t w = Num<T>::from2(exp2f(s[mt][2 * h] - base), exp2f(s[mt][2 * h + 1] - base));
        const float2 used = Num<T>::to2(w);
        sum[mt][h] = fmaf(sum[mt][h], shrink, used.x + used.y);
        const uint32_t at = weights + piece<64>(r, warp) * 16 + 4 * t4;
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(w) : "memory");
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          o[mt][j][2 * h] *= shrink;
          o[mt][j][2 * h + 1] *= shrink;
        }
      }
    }
    // A row's weight of a key that it does not see is 0, but 0 times an infinite or NaN value is not:
    // where rows differ in what they see and a value of the tile is not finite, the products are
    // formed one by one, the unseen ones left out.
    bool one_by_one = false;
    if (edge && cur.news > 1) {
      bool odd = false;
      for (int x = tid; x < kKvTile * kPieces; x += kThreads) {
        const uint4 v = *reinterpret_cast<const uint4*>(smem + (values - ring) + x * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = (&v.x)[e], lo = Num<T>::kExponent & 0xffffu, hi = Num<T>::kExponent & 0xffff0000u;
          odd = odd || (w & lo) == lo || (w & hi) == hi;
        }
      }
      one_by_one = __syncthreads_or(odd);
    } else {
      __syncthreads();
    }
    if (!one_by_one) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {               // 32 keys at a time
        uint32_t vf[kCols][4];
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          if (kPieces % kWarps == 0 || j * kWarps + warp < kPieces)
            ldm_x4_trans(vf[j], values + piece<D>(kk * 32 + lane, j * kWarps + warp) * 16);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if (MT > 1 && mt >= row_tiles) continue;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t wf[4];
            ldm_x4(wf, weights + piece<64>(mt * 16 + (lane & 15), kk * 4 + k * 2 + (lane >> 4)) * 16);
#pragma unroll
            for (int j = 0; j < kCols; ++j)
              if (kPieces % kWarps == 0 || j * kWarps + warp < kPieces)
                mma(T(), o[mt][j], wf, vf[j][2 * k], vf[j][2 * k + 1]);
          }
        }
      }
    } else {
      const unsigned short* wts = reinterpret_cast<const unsigned short*>(smem + (weights - ring));
      const unsigned short* val = reinterpret_cast<const unsigned short*>(smem + (values - ring));
#pragma unroll 1
      for (int k = 0; k < kKvTile; ++k) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          const int c = j * kWarps + warp;
          if (c >= kPieces) continue;
          const uint32_t pair = *reinterpret_cast<const uint32_t*>(val + piece<D>(k, c) * 8 + 2 * t4);
          const float2 v = Num<T>::to2(pair);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int last = upto[mt][h];
              if (mt >= row_tiles || k0 + k > last || last - (k0 + k) >= reach) continue;
              const float w = Num<T>::to1(wts[piece<64>(mt * 16 + g + 8 * h, k >> 3) * 8 + (k & 7)]);
              o[mt][j][2 * h] = fmaf(w, v.x, o[mt][j][2 * h]);
              o[mt][j][2 * h + 1] = fmaf(w, v.y, o[mt][j][2 * h + 1]);
            }
          }
        }
      }
    }

    const bool item_ends = cur.tile + 1 == cur.tiles;
    if (item_ends || i + 1 == n_tiles) {
      // sums over the warps' keys
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (MT > 1 && mt >= row_tiles) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = sum[mt][h];
          x += __shfl_xor_sync(~0u, x, 1);
          x += __shfl_xor_sync(~0u, x, 2);
          if (t4 == 0) maxima[(mt * 16 + g + 8 * h) * kWarps + warp] = x;
        }
      }
      __syncthreads();
      const bool whole = piece_start == 0 && item_ends;
      const int row0 = cur.block * S::kRows, rows = min(S::kRows, cur.news * V.group - row0);
      // a piece that began before this CTA's run, or one that goes on behind it
      float* part = V.partials + (size_t)(2 * blockIdx.x + (piece_start == 0)) * S::kRows * (D + 2);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = mt * 16 + g + 8 * h;
          if (r >= rows) continue;
          const float4 x = *reinterpret_cast<const float4*>(maxima + r * kWarps);
          const float4 y = *reinterpret_cast<const float4*>(maxima + r * kWarps + 4);
          const float all = ((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w));
          if (whole) {
            const int t = (row0 + r) / V.group, head = cur.head * V.group + row0 + r - t * V.group;
            T* out = reinterpret_cast<T*>(a.out) + (((int64_t)cur.b * V.max_new + t) * V.n_heads + head) * D;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
              const int c = j * kWarps + warp;
              if (c < kPieces)
                *reinterpret_cast<uint32_t*>(out + c * 8 + 2 * t4) = Num<T>::from2(o[mt][j][2 * h] / all, o[mt][j][2 * h + 1] / all);
            }
          } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
              const int c = j * kWarps + warp;
              if (c < kPieces)
                *reinterpret_cast<float2*>(part + (size_t)r * D + c * 8 + 2 * t4) = make_float2(o[mt][j][2 * h], o[mt][j][2 * h + 1]);
            }
            if (warp == 0 && t4 == 0) {
              part[S::kRows * D + r] = m[mt][h];
              part[S::kRows * (D + 1) + r] = all;
            }
          }
        }
      }
    }
    stage = stage + 1 == S::kStages ? 0 : stage + 1;
    cur.step(V);
  }
}

// Finishes the heads that the runs' ends cut: a CTA per head and row, lanes along the columns, the
// pieces dealt to the thread groups and joined in a fixed order.  Bound: latency.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv_join_kernel(KvView V, void* out) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes;
  __shared__ float4 fold[kGroups][kLanes];
  pdl_wait();
  const int n = V.counts[KV_JOINS], R = V.rows_per_block;
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const size_t slot = (size_t)R * (D + 2);
  for (int u = blockIdx.x; u < n * R; u += gridDim.x) {
    const int4 join = V.joins[u / R];
    const int r = u % R, news = V.seq_plan[join.z].z;
    const int blocks = kv_row_blocks(news, V.group, R), head = join.w / blocks, row = (join.w - head * blocks) * R + r;
    if (row >= news * V.group) continue;           // (the same for the whole CTA)
    const int pieces = join.y - join.x + 1;
    // piece p: the first CTA's second slot, every other one's first
    auto at = [&](int p) { return V.partials + (size_t)(2 * (join.x + p) + (p == 0)) * slot; };
    float top = -INFINITY;                         // every warp by itself
    for (int p = threadIdx.x & 31; p < pieces; p += 32) top = fmaxf(top, at(p)[R * D + r]);
#pragma unroll
    for (int k = 16; k; k /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, k));
    const float base = top == -INFINITY ? 0.f : top;
    float all = 0.f;
    for (int p = threadIdx.x & 31; p < pieces; p += 32)
      all = fmaf(at(p)[R * (D + 1) + r], exp2f(at(p)[R * D + r] - base), all);
#pragma unroll
    for (int k = 16; k; k /= 2) all += __shfl_xor_sync(~0u, all, k);
    if (group < kGroups) {
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int p = group; p < pieces; p += kGroups) {
        const float w = exp2f(at(p)[R * D + r] - base);
        const float4 x = *reinterpret_cast<const float4*>(at(p) + (size_t)r * D + 4 * lane);
        acc.x = fmaf(w, x.x, acc.x);
        acc.y = fmaf(w, x.y, acc.y);
        acc.z = fmaf(w, x.z, acc.z);
        acc.w = fmaf(w, x.w, acc.w);
      }
      fold[group][lane] = acc;
    }
    __syncthreads();
    if (group == 0) {
      float4 acc = fold[0][lane];
#pragma unroll
      for (int k = 1; k < kGroups; ++k) {
        const float4 x = fold[k][lane];
        acc.x += x.x;
        acc.y += x.y;
        acc.z += x.z;
        acc.w += x.w;
      }
      const int t = row / V.group;
      T* to = reinterpret_cast<T*>(out) +
              (((int64_t)join.z * V.max_new + t) * V.n_heads + head * V.group + row - t * V.group) * D + 4 * lane;
      *reinterpret_cast<uint2*>(to) = make_uint2(Num<T>::from2(acc.x / all, acc.y / all), Num<T>::from2(acc.z / all, acc.w / all));
    }
    __syncthreads();
  }
}

// What to do with the kernels for a type, head dimension and row tiles.
template <typename T, int D, int MT, typename F>
cudaError_t with(F f) {
  return f(kv_attention_kernel<T, D, MT>, kv_join_kernel<T, D>, Shape<D, MT>::kSmem);
}
template <typename T, int D, typename F>
cudaError_t with_rows(int row_tiles, F f) {
  if (row_tiles == 1) return with<T, D, 1>(f);
  if (row_tiles == 2) return with<T, D, 2>(f);
  if (row_tiles == 4) return with<T, D, 4>(f);
  if constexpr (D <= 128) return with<T, D, 8>(f);
  return cudaErrorInvalidValue;
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
cudaError_t with_kernels(const lif_kv* kv, F f) {
  const lif_kv_desc& d = kv->desc;
  return d.dtype == LIF_TYPE_F16 ? with_dim<__half>(d.head_dim, kv->row_tiles, f)
                                 : with_dim<__nv_bfloat16>(d.head_dim, kv->row_tiles, f);
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

cudaError_t kv_attention_configure(const lif_kv* kv, int* ctas_per_sm) {
  return with_kernels(kv, [&](auto kernel, auto, int smem) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, kernel, kThreads, smem);
    return e;
  });
}

cudaError_t launch_kv_attention(const lif_kv* kv, int layer, const void* q, void* out, cudaStream_t st) {
  const lif_kv_desc& d = kv->desc;
  AttendArgs a;
  a.q = q;
  a.out = out;
  a.pages = (const char*)d.dev_pages + (size_t)layer * d.n_pages * kv_page_elems(d) * 2;
  a.scale_log2 = kv->scale * 1.4426950408889634f;
  return with_kernels(kv, [&](auto kernel, auto join, int smem) {
    cudaError_t e = launch_k(kernel, dim3(kv->v.ctas), dim3(kThreads), smem, st, 1, kv->v, a);
    if (e == cudaSuccess) e = launch_k(join, dim3(2 * kv->n_sm), dim3(kThreads), 0, st, 1, kv->v, out);
    return e;
  });
}

}  // namespace lif
