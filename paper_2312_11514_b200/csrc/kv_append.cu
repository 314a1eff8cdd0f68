// The new tokens' queries, keys and values on their way to attention, in one pass: norm of every
// query and key head, rotation by position, keys and values into their pages.
//
//   norm      y = x / sqrt(mean(x^2) + eps) * w      or  (x - mean) / sqrt(var + eps) * w + b
//   rotation  (u, v) -> s (u cos a - v sin a, u sin a + v cos a),  a = position * f_i
//
// A group of lanes holds a head's row, 8 elements a lane (one 16-byte load), so both sums of a norm
// are shuffles inside the group and the row is read and written once.  A CTA works on one token: the
// cosines and sines of its position are computed once, laid out as each lane's elements need them, and serve
// all rows that its groups take in turn; the next row travels while one is worked on.
// The angle is a fraction of a turn in 64-bit integer arithmetic (position * f mod 2^64): exact to
// 2^-34 of a turn at position 2^30, where an fp32 product would be off by whole turns; sincospif then
// takes the fraction, reduced, in fp32.  Norm and rotation are fp32; one rounding at the end.
// Bound: latency for a decode step's few tokens (3.1 us for 8 tokens of 192 rows of 64: length and page are
// two dependent round trips, the rows travel beside the second); latency too for long pieces of a prompt, where half
// of the stalls are loads and 37% of the issue slots are used: queries are fetched one row ahead, keys and
// values past a group's first not at all (25 MB in 7.4 us, 52% of measured HBM; the first version took 9.0).
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

constexpr int kAppendThreads = 64;

template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(KvView V, AppendArgs a) {
  constexpr int kLanes = D / 8;                                          // lanes that hold elements
  constexpr int kGroup = D <= 64 ? 8 : D <= 128 ? 16 : 32;               // lanes of a row
  constexpr int kRows = kAppendThreads / kGroup;
  __shared__ float2 turn[D / 2];                                         // cos, sin
  __shared__ __align__(16) float normed[kRows][D + 4];
  const int token = blockIdx.x, b = token / V.max_new, t = token - b * V.max_new;
  const int group = threadIdx.x / kGroup, lane = threadIdx.x % kGroup;
  const bool holds = lane < kLanes;
  const unsigned live = kGroup == 32 ? ~0u : ((1u << kGroup) - 1u) << (threadIdx.x & 31 & ~(kGroup - 1));   // the group's lanes
  pdl_wait();
  const int news = V.n_new[b], pos = V.lens[b] - news + t;
  if (t >= news) return;
  // Rows are dealt to the groups in the order queries, keys, values: this group's first of each.
  const int stride = gridDim.y * kRows, first = blockIdx.y * kRows + group;
  auto next_from = [&](int at) { return first + (at - first + stride - 1) / stride * stride - at; };
  const int first_k = first >= V.n_heads ? first - V.n_heads : next_from(V.n_heads);
  const int first_v = first >= V.n_heads + V.n_kv_heads ? first - V.n_heads - V.n_kv_heads : next_from(V.n_heads + V.n_kv_heads);
  auto source = [&](const lif_kv_rows& r, int h) {
    return reinterpret_cast<const T*>(r.dev) + (int64_t)token * r.token_stride + h * r.head_stride + 8 * lane;
  };
  const uint4 none = make_uint4(0, 0, 0, 0);
  auto fetch = [&](const T* p, bool there) { return there && holds ? *reinterpret_cast<const uint4*>(p) : none; };
  // What the token's first rows need is on its way at once: the rows, the page, the frequencies.
  const T* src = source(a.q, first);
  uint4 raw = fetch(src, first < V.n_heads);
  const uint4 raw_k = fetch(source(a.k, first_k), first_k < V.n_kv_heads);
  const uint4 raw_v = fetch(source(a.v, first_v), first_v < V.n_kv_heads);
  const int page = V.table[(size_t)b * V.max_pages + (pos >> V.page_shift)];
  if (a.rope != LIF_ROPE_NONE) {
    for (int i = threadIdx.x; i < a.rope_dims / 2; i += kAppendThreads) {
      const uint64_t part = V.turns[i] * (uint64_t)pos;
      float s, c;
      sincospif((float)(int32_t)(part >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
      turn[i] = make_float2(c * a.rope_scale, s * a.rope_scale);
    }
  }
  __syncthreads();
  // A rotated element is x c + (its partner) s, the sine's sign that of its place in the pair; the same
  // for every row of the token.
  const int half = a.rope_dims / 2;
  float cosines[8], sines[8];
  int partner[8];
  unsigned rotates = 0;
  if (a.rope != LIF_ROPE_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = 8 * lane + i;
      if (e >= a.rope_dims) continue;
      const bool second = a.rope == LIF_ROPE_HALF ? e >= half : i & 1;
      const float2 c = turn[a.rope == LIF_ROPE_HALF ? (second ? e - half : e) : e / 2];
      cosines[i] = c.x;
      sines[i] = second ? c.y : -c.y;
      partner[i] = second ? e - half : e + half;
      rotates |= 1u << i;
    }
  }
  // norm and rotation of a row
  auto turned = [&](const uint4& in, const uint4& weight, const uint4& bias, bool biased) {
    float x[8];
    const uint32_t* w = &in.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = Num<T>::to2(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
    if (a.norm != LIF_NORM_NONE) {
      if (a.norm == LIF_NORM_LAYER) {
        float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
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
      const float inv = rsqrtf(s * (1.f / D) + a.eps);
      const uint32_t *wp = &weight.x, *bp = &bias.x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = Num<T>::to2(wp[i]);
        x[2 * i] *= inv * f.x;
        x[2 * i + 1] *= inv * f.y;
        if (biased) {
          const float2 g = Num<T>::to2(bp[i]);
          x[2 * i] += g.x;
          x[2 * i + 1] += g.y;
        }
      }
    }
    if (a.rope == LIF_ROPE_INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        if (rotates >> i & 1) {
          const float u = x[i], v = x[i + 1];
          x[i] = fmaf(v, sines[i], u * cosines[i]);
          x[i + 1] = fmaf(u, sines[i + 1], v * cosines[i + 1]);
        }
    } else if (a.rope == LIF_ROPE_HALF) {
      float4* to = reinterpret_cast<float4*>(normed[group] + 8 * lane);
      if (holds) {
        to[0] = make_float4(x[0], x[1], x[2], x[3]);
        to[1] = make_float4(x[4], x[5], x[6], x[7]);
      }
      __syncwarp(live);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (rotates >> i & 1) x[i] = fmaf(normed[group][partner[i]], sines[i], x[i] * cosines[i]);
      __syncwarp(live);
    }
    return make_uint4(Num<T>::from2(x[0], x[1]), Num<T>::from2(x[2], x[3]), Num<T>::from2(x[4], x[5]), Num<T>::from2(x[6], x[7]));
  };
  const bool plain = a.norm == LIF_NORM_NONE && a.rope == LIF_ROPE_NONE;   // rows pass as they came
  auto affine = [&](const void* p) { return fetch(reinterpret_cast<const T*>(p) + 8 * lane, p != nullptr); };

  if (first < V.n_heads) {
    const bool biased = a.norms.dev_q_bias != nullptr;
    const uint4 weight = affine(a.norms.dev_q_weight), bias = affine(a.norms.dev_q_bias);
    T* dst = reinterpret_cast<T*>(a.q_out) + ((size_t)token * V.n_heads + first) * D + 8 * lane;
    const int64_t step = (int64_t)stride * a.q.head_stride;
    for (int h = first; h < V.n_heads; h += stride) {
      const uint4 now = raw;
      src += step;
      raw = fetch(src, h + stride < V.n_heads);            // the next row's load runs beside this row's work
      const uint4 out = plain ? now : turned(now, weight, bias, biased);
      if (holds) *reinterpret_cast<uint4*>(dst) = out;
      dst += (size_t)stride * D;
    }
  }
  // keys and values: [page][key, value][head][row in the page]
  T* rows = reinterpret_cast<T*>(a.pages) + (((size_t)page * 2 * V.n_kv_heads << V.page_shift) + (pos & ((1 << V.page_shift) - 1))) * D + 8 * lane;
  if (first_k < V.n_kv_heads) {
    const bool biased = a.norms.dev_k_bias != nullptr;
    const uint4 weight = affine(a.norms.dev_k_weight), bias = affine(a.norms.dev_k_bias);
    for (int h = first_k; h < V.n_kv_heads; h += stride) {
      const uint4 now = h == first_k ? raw_k : fetch(source(a.k, h), true);
      const uint4 out = plain ? now : turned(now, weight, bias, biased);
      if (holds) *reinterpret_cast<uint4*>(rows + ((size_t)h << V.page_shift) * D) = out;
    }
  }
  for (int h = first_v; h < V.n_kv_heads; h += stride) {
    const uint4 now = h == first_v ? raw_v : fetch(source(a.v, h), true);
    if (holds) *reinterpret_cast<uint4*>(rows + ((size_t)(V.n_kv_heads + h) << V.page_shift) * D) = now;
  }
}

template <typename T, int D>
cudaError_t launch(const lif_kv* kv, const AppendArgs& a, cudaStream_t st) {
  const KvView& v = kv->v;
  const int rows_at_once = kAppendThreads / (D <= 64 ? 8 : D <= 128 ? 16 : 32);
  const int tokens = v.max_seqs * v.max_new, rows = v.n_heads + 2 * v.n_kv_heads;
  // Two warps a CTA and many rows a group: what a token's rows share (angles, weights) is laid out once for
  // all of them.  1024 tokens of 48 rows of 128: 7.4 us; four warps 8.1, eight 10.4, one 10.0.  Where tokens
  // alone leave SMs idle, more CTAs a token, while that keeps the grid within five CTAs a SM (64 tokens of 96
  // rows: 3.8 us, within two a SM 4.5, within sixteen 4.7).
  int per_token = (rows + rows_at_once - 1) / rows_at_once;
  const int room = (5 * kv->n_sm + tokens - 1) / tokens;
  if (per_token > room) per_token = room;
  return launch_k(kv_append_kernel<T, D>, dim3(tokens, per_token), dim3(kAppendThreads), 0, st, 1, v, a);
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
