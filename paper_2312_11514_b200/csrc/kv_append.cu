// The new tokens' queries, keys and values on their way to attention, in one pass: norm of every
// query and key head, rotation by position, keys and values into their pages.
//
//   norm      y = x / sqrt(mean(x^2) + eps) * w      or  (x - mean) / sqrt(var + eps) * w + b
//   rotation  (u, v) -> s (u cos a - v sin a, u sin a + v cos a),  a = position * f_i
//
// A group of lanes holds a head's row, 8 elements a lane (one 16-byte load), so both sums of a norm
// are shuffles inside the group and the row is read and written once.  A CTA works on one token: the
// cosines and sines of its position are computed once, into shared memory, and serve all its heads.
// The angle is a fraction of a turn in 64-bit integer arithmetic (position * f mod 2^64): exact to
// 2^-34 of a turn at position 2^30, where an fp32 product would be off by whole turns; sincospif then
// takes the fraction, reduced, in fp32.  Norm and rotation are fp32; one rounding at the end.
// Bound: latency for a decode step's few tokens (the row's load runs beside those of length, page id
// and frequencies), HBM for long pieces of a prompt.
#include "kv_internal.cuh"

namespace lif {
namespace {

struct AppendArgs {
  lif_kv_rows q, k, v;
  lif_kv_norms norms;
  void *q_out, *pages;               // pages: this layer's
  float eps, rope_scale;
  int norm, rope, rope_dims;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(KvView V, AppendArgs a) {
  constexpr int kLanes = D / 8;                                          // lanes that hold elements
  constexpr int kGroup = D <= 64 ? 8 : D <= 128 ? 16 : 32;               // lanes of a row
  constexpr int kRows = kThreads / kGroup;
  __shared__ float2 turn[D / 2];                                         // cos, sin
  __shared__ float normed[kRows][D + 4];
  const int token = blockIdx.x, b = token / V.max_new, t = token - b * V.max_new;
  const int group = threadIdx.x / kGroup, lane = threadIdx.x % kGroup;
  const bool holds = lane < kLanes;
  pdl_wait();
  const int news = V.n_new[b], pos = V.lens[b] - news + t;
  if (t >= news) return;
  if (a.rope != LIF_ROPE_NONE) {
    for (int i = threadIdx.x; i < a.rope_dims / 2; i += kThreads) {
      const uint64_t part = V.turns[i] * (uint64_t)pos;
      float s, c;
      sincospif((float)(int32_t)(part >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
      turn[i] = make_float2(c * a.rope_scale, s * a.rope_scale);
    }
  }
  const int page = V.table[(size_t)b * V.max_pages + (pos >> V.page_shift)];
  const int row_in_page = pos & ((1 << V.page_shift) - 1);
  __syncthreads();
  const int rows = V.n_heads + 2 * V.n_kv_heads;
  for (int r = blockIdx.y * kRows + group; r < rows; r += gridDim.y * kRows) {
    const int kind = r < V.n_heads ? 0 : r < V.n_heads + V.n_kv_heads ? 1 : 2;   // query, key, value
    const int h = kind == 0 ? r : r - V.n_heads - (kind == 2 ? V.n_kv_heads : 0);
    const lif_kv_rows& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (holds)
      raw = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(src.dev) + (int64_t)token * src.token_stride +
                                            h * src.head_stride + 8 * lane);
    T* dst = kind == 0 ? reinterpret_cast<T*>(a.q_out) + ((size_t)token * V.n_heads + h) * D
                       : reinterpret_cast<T*>(a.pages) +
                             ((((size_t)page * 2 + kind - 1) * V.n_kv_heads + h << V.page_shift) + row_in_page) * D;
    if (kind < 2) {
      float x[8];
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = Num<T>::to2(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
      // the lanes of this group that are in this turn of the loop (the last one may lack groups)
      const unsigned live = kGroup == 32 ? ~0u : ((1u << kGroup) - 1u) << (threadIdx.x & 31 & ~(kGroup - 1));
      if (a.norm != LIF_NORM_NONE) {
        if (a.norm == LIF_NORM_LAYER) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) s += x[i];
#pragma unroll
          for (int o = kGroup / 2; o; o /= 2) s += __shfl_xor_sync(live, s, o);
          s *= 1.f / D;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = holds ? x[i] - s : 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
#pragma unroll
        for (int o = kGroup / 2; o; o /= 2) s += __shfl_xor_sync(live, s, o);
        const float inv = 1.f / sqrtf(s * (1.f / D) + a.eps);
        const T* weight = reinterpret_cast<const T*>(kind == 0 ? a.norms.dev_q_weight : a.norms.dev_k_weight);
        const T* bias = reinterpret_cast<const T*>(kind == 0 ? a.norms.dev_q_bias : a.norms.dev_k_bias);
        if (holds) {
          const uint4 wv = *reinterpret_cast<const uint4*>(weight + 8 * lane);
          const uint4 bv = bias ? *reinterpret_cast<const uint4*>(bias + 8 * lane) : make_uint4(0, 0, 0, 0);
          const uint32_t *wp = reinterpret_cast<const uint32_t*>(&wv), *bp = reinterpret_cast<const uint32_t*>(&bv);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = Num<T>::to2(wp[i]), g = Num<T>::to2(bp[i]);
            x[2 * i] = fmaf(x[2 * i] * inv, f.x, g.x);
            x[2 * i + 1] = fmaf(x[2 * i + 1] * inv, f.y, g.y);
          }
        }
      }
      if (a.rope == LIF_ROPE_INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (8 * lane + 2 * i < a.rope_dims) {
            const float2 c = turn[4 * lane + i];
            const float u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * c.x - v * c.y;
            x[2 * i + 1] = u * c.y + v * c.x;
          }
      } else if (a.rope == LIF_ROPE_HALF) {
        const int half = a.rope_dims / 2;
        if (holds) {
#pragma unroll
          for (int i = 0; i < 8; ++i) normed[group][8 * lane + i] = x[i];
        }
        __syncwarp(live);
        if (holds) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = 8 * lane + i;
            if (e < half) {
              const float2 c = turn[e];
              x[i] = x[i] * c.x - normed[group][e + half] * c.y;
            } else if (e < a.rope_dims) {
              const float2 c = turn[e - half];
              x[i] = normed[group][e - half] * c.y + x[i] * c.x;
            }
          }
        }
        __syncwarp(live);
      }
      if (a.norm != LIF_NORM_NONE || a.rope != LIF_ROPE_NONE) {          // otherwise as it came
        uint32_t* o = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = Num<T>::from2(x[2 * i], x[2 * i + 1]);
      }
    }
    if (holds) *reinterpret_cast<uint4*>(dst + 8 * lane) = raw;
  }
}

template <typename T, int D>
cudaError_t launch(const lif_kv* kv, const AppendArgs& a, cudaStream_t st) {
  const KvView& v = kv->v;
  const int rows_at_once = kThreads / (D <= 64 ? 8 : D <= 128 ? 16 : 32);
  const int tokens = v.max_seqs * v.max_new, rows = v.n_heads + 2 * v.n_kv_heads;
  // As many CTAs per token as give every head's row a group of its own, while that keeps the grid
  // within two CTAs a SM; where there are more tokens a CTA takes several rows in turn and its
  // cosines serve them all.
  int per_token = (rows + rows_at_once - 1) / rows_at_once;
  const int room = (2 * kv->n_sm + tokens - 1) / tokens;
  if (per_token > room) per_token = room;
  return launch_k(kv_append_kernel<T, D>, dim3(tokens, per_token), dim3(kThreads), 0, st, 1, v, a);
}

template <typename T>
cudaError_t launch_dim(const lif_kv* kv, const AppendArgs& a, cudaStream_t st) {
  switch (kv->desc.head_dim) {
    case 64: return launch<T, 64>(kv, a, st);
    case 80: return launch<T, 80>(kv, a, st);
    case 96: return launch<T, 96>(kv, a, st);
    case 128: return launch<T, 128>(kv, a, st);
    default: return launch<T, 256>(kv, a, st);
  }
}

}  // namespace

cudaError_t launch_kv_append(const lif_kv* kv, int layer, const lif_kv_rows& q, const lif_kv_rows& k,
                             const lif_kv_rows& v, const lif_kv_norms& norms, void* q_out, cudaStream_t st) {
  const lif_kv_desc& d = kv->desc;
  AppendArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.norms = norms;
  a.q_out = q_out;
  a.pages = (char*)d.dev_pages + (size_t)layer * d.n_pages * kv_page_elems(d) * 2;
  a.eps = d.norm_eps;
  a.rope_scale = d.rope_scale;
  a.norm = d.norm;
  a.rope = d.rope;
  a.rope_dims = d.rope_dims;
  return d.dtype == LIF_TYPE_F16 ? launch_dim<__half>(kv, a, st) : launch_dim<__nv_bfloat16>(kv, a, st);
}

}  // namespace lif
