// Paged key-value cache: argument checks, workspace, and the kernels that change its tables.
//
// The tables are device state, as the neuron window's are: a step's page needs, a beam's reordering
// or a compaction are known only on the device, and no size returns to the host, so one captured
// graph serves every token.  What bounds these kernels is latency (dependent round trips over a few
// kilobytes of tables), except kv_copy_pages_kernel, which moves pages and is bound by HBM.
//
//   kv_reserve_kernel   once per token: one CTA, a thread per place, so that everything a place
//                       decides sits in its thread and the shared parts are two block scans; three
//                       round trips (lengths; last pages and the first free ones; references)
//   kv_arrange_kernel   fork and load: tables of up to kSmallPages pages and kSmallTable entries in one
//                       CTA, references counted in shared memory; larger ones in a cluster of eight, whose
//                       barrier separates the phases in place of launches (64 places of ten pages,
//                       loaded and compacted: 28 us in clusters, 15 us so)
//   kv_compact_kernel   likewise (kv_compact_small_kernel: one CTA, lists and new ids in shared memory)
//   kv_copy_pages_kernel  what reserve and compact decided to copy, all layers; a warp per 4 KB
//
// Free pages are given out lowest id first, references are counted (integer sums, whatever order),
// so the same calls give the same tables.
#include <cooperative_groups.h>
#include <math.h>
#include <string.h>

#include <new>

#include "kv_internal.cuh"

namespace lif {
namespace {

namespace cg = cooperative_groups;

__device__ void kv_refuse(const KvView& v, int code) {
  atomicCAS(v.counts + LIF_KV_CNT_STATUS, LIF_OK, code);
  v.counts[LIF_KV_CNT_REFUSED] += 1;
}

// Exclusive sum over the block's kKvPlanThreads threads; *total: the whole.  Ends with a barrier.
__device__ unsigned long long block_scan(unsigned long long x, unsigned long long* total) {
  __shared__ unsigned long long warp_sum[kKvPlanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long s = x;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned long long y = __shfl_up_sync(~0u, s, o);
    if (lane >= o) s += y;
  }
  if (lane == 31) warp_sum[warp] = s;
  __syncthreads();
  if (warp == 0) {
    unsigned long long w = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const unsigned long long y = __shfl_up_sync(~0u, w, o);
      if (lane >= o) w += y;
    }
    warp_sum[lane] = w;
  }
  __syncthreads();
  const unsigned long long before = (warp ? warp_sum[warp - 1] : 0) + s - x;
  *total = warp_sum[kKvPlanThreads / 32 - 1];
  __syncthreads();
  return before;
}

// The work of the step's attention calls, the same for every layer: tiles of kKvTile keys, in the
// order place, key-value head, row block, tile, cut into shares, one a CTA.  Short work (kLongRun tiles
// a share at most) is done so; of a longer share 85 % are the CTA's first run, and what remains
// is cut into further runs of a 24th of a share, which CTAs take as they become free.  Runs are
// numbered as they lie.  Thread b holds place b's tokens.  A head and row block that the end of a run
// cuts is entered in `joins`.  Three quarters and twentieths take 1 % more time (more pieces to join), nine tenths
// and 30ths as much for one long sequence but 2 % more for a batch (too little to share out).
constexpr int kLongRun = 15;
__device__ void kv_plan(const KvView& v, int tokens, int n_new) {
  __shared__ int first[kKvPlanThreads];
  __shared__ int4 place[kKvPlanThreads];
  __shared__ int n_joins;
  const int b = threadIdx.x;
  if (b == 0) n_joins = 0;
  const int nt = b < v.max_seqs ? kv_tiles(tokens, n_new, v.window) : 0;
  unsigned long long all;
  const int at = (int)block_scan(
      (unsigned long long)nt * v.n_kv_heads * kv_row_blocks(n_new, v.group, v.rows_per_block), &all);
  const int total = (int)all;
  first[b] = b < v.max_seqs ? at : 0x7fffffff;
  place[b] = make_int4(at, tokens, n_new, nt);
  if (b < v.max_seqs) v.seq_plan[b] = place[b];
  __syncthreads();
  const int share = (total - 1) / v.ctas + 1;        // (total = 0: 1, and no run)
  const int shares = (total + share - 1) / share;
  int q0 = share, q1 = share, more = 0, n_more = 0;
  if (share > kLongRun && v.max_runs >= 6 * v.ctas) {
    q0 = (int)(17LL * share / 20);
    q1 = (share + 23) / 24;                          // share - q0 <= 5 q1: six runs a share at most
    more = (share - q0 + q1 - 1) / q1;
    const int rest = total - (shares - 1) * share - q0;
    n_more = (shares - 1) * more + (rest > 0 ? (rest + q1 - 1) / q1 : 0);
  }
  const int runs = shares ? (shares - 1) * (1 + more) + 1 + n_more - (shares - 1) * more : 0;
  auto begin_of = [&](int run) {
    const int c = run / (1 + more), j = run - c * (1 + more);
    return c * share + (j ? q0 + (j - 1) * q1 : 0);
  };
  auto run_of = [&](int tile) {
    const int c = tile / share, in = tile - c * share;
    return c * (1 + more) + (in < q0 ? 0 : 1 + (in - q0) / q1);
  };
  for (int c = b; c < runs; c += kKvPlanThreads) {
    const int g = begin_of(c);
    int lo = 0, hi = v.max_seqs;              // last place whose first tile is <= g
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first[mid] <= g) lo = mid; else hi = mid;
    }
    const int4 p = place[lo];
    const int in = c % (1 + more), share_of = c / (1 + more);
    v.run_plan[in ? v.ctas + share_of * more + in - 1 : share_of] = make_int4(lo, p.x, p.y, p.z);
    const int item = (g - p.x) / p.w, s = p.x + item * p.w;
    if (s < g && begin_of(c - 1) <= s) {      // the first run that begins inside the item
      const int blocks = kv_row_blocks(p.z, v.group, v.rows_per_block), head = item / blocks;
      // (where an entry stands does not matter)
      v.joins[atomicAdd(&n_joins, 1)] = make_int4((c - 1) | run_of(s + p.w - 1) << 16, lo, head << 16 | (item - head * blocks), p.z);
    }
  }
  __syncthreads();
  if (b == 0) {
    v.counts[KV_TILES] = total;
    v.counts[KV_SHARES] = shares;
    v.counts[KV_SHARE] = share;
    v.counts[KV_FIRST_TILES] = q0;
    v.counts[KV_MORE_TILES] = q1;
    v.counts[KV_MORE] = more;
    v.counts[KV_MORE_IN_ALL] = n_more;
    v.counts[KV_JOINS] = n_joins;
    v.counts[KV_TAKEN] = 0;
  }
}

// Pages that a step can take: its tokens' and one for a copy, a place.
static_assert(LIF_KV_MAX_SEQS <= kKvPlanThreads, "");
int reserve_list(const KvView& v) {
  const int n = v.max_seqs * ((v.max_new >> v.page_shift) + 2);
  return n > kKvPlanThreads ? n : kKvPlanThreads;
}
constexpr int kReserveListMost = kKvPlanThreads * (LIF_KV_MAX_NEW / 8 + 2);

__global__ void __launch_bounds__(kKvPlanThreads)
kv_reserve_kernel(KvView v, const int32_t* n_new) {
  extern __shared__ int page_list[];         // [reserve_list]
  pdl_wait();
  const int b = threadIdx.x;
  const bool mine = b < v.max_seqs;
  const int tokens = mine ? v.lens[b] : 0, n = mine ? n_new[b] : 0;
  const int n_free = v.counts[LIF_KV_CNT_FREE], free_from = v.counts[KV_FREE_FROM];
  const bool bad = n < 0 || n > v.max_new;
  const int used = kv_pages_of(tokens, v.page_shift), wanted = kv_pages_of(tokens + (bad ? 0 : n), v.page_shift);
  const int filled = tokens & ((1 << v.page_shift) - 1);
  int tail = -1, holders = 0;
  if (!bad && n > 0 && filled) tail = v.table[(size_t)b * v.max_pages + used - 1];
  // the first four times kKvPlanThreads pages that may be free: on their way beside the last pages
  auto free_of = [&](int p) {
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < v.n_pages && v.refs[p + i] == 0) mask |= 1u << i;
    return mask;
  };
  int p0 = free_from & ~3;
  unsigned free4 = free_of(p0 + 4 * b);
  if (tail >= 0) holders = v.refs[tail];
  // Copy on write.  A page that several entries name and that this place is about to write behind
  // its own rows; the lowest place may go on in it where nobody is left who does not leave it.
  bool copy = holders > 1;
  page_list[b] = copy ? tail : -1;
  if (__syncthreads_or(copy) && copy) {
    int growers = 0, lowest = b;
    for (int o = 0; o < v.max_seqs; ++o)
      if (page_list[o] == tail) {
        ++growers;
        lowest = o < lowest ? o : lowest;
      }
    copy = !(growers == holders && lowest == b);
  }
  // one scan: pages (up to 10 a place), copies, and what refuses the call
  const int take = wanted - used + copy;
  unsigned long long sums;
  const unsigned long long before =
      block_scan((unsigned long long)take | (unsigned long long)copy << 16 | (unsigned long long)(wanted > v.max_pages) << 32 |
                     (unsigned long long)bad << 48, &sums);
  const int total = (int)(sums & 0xffff), n_copies = (int)(sums >> 16 & 0xffff);
  const int at = (int)(before & 0xffff), copy_at = (int)(before >> 16 & 0xffff);
  int code = sums >> 48 ? LIF_ERR_INVALID_ARG : (sums >> 32 & 0xffff) || total > n_free ? LIF_ERR_CAPACITY : LIF_OK;
  // the `total` lowest free pages, four a thread and round
  if (code == LIF_OK && total > 0) {
    int found = 0;
    for (;;) {
      unsigned long long here;
      int r = found + (int)block_scan(__popc(free4), &here);
      const int p = p0 + 4 * b;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (free4 >> i & 1) {
          if (r < total) page_list[r] = p + i;
          ++r;
        }
      found += (int)here;
      p0 += 4 * kKvPlanThreads;
      if (found >= total || p0 >= v.n_pages) break;
      free4 = free_of(p0 + 4 * b);
    }
    __syncthreads();
    if (found < total) code = LIF_ERR_STATE;
  }
  if (code != LIF_OK) {
    if (mine) v.n_new[b] = 0;
    if (b == 0) {
      kv_refuse(v, code);
      v.counts[LIF_KV_CNT_COPIES] = 0;
    }
    kv_plan(v, tokens, 0);
    return;
  }
  if (mine) {
    int next = at;
    if (copy) {
      const int page = page_list[next++];
      v.table[(size_t)b * v.max_pages + used - 1] = page;
      v.list_a[copy_at] = tail;
      v.list_b[copy_at] = page;
      v.copy_tokens[copy_at] = filled;
      atomicSub(v.refs + tail, 1);
      v.refs[page] = 1;
    }
    for (int j = used; j < wanted; ++j) {
      const int page = page_list[next++];
      v.table[(size_t)b * v.max_pages + j] = page;
      v.refs[page] = 1;
    }
    v.lens[b] = tokens + n;
    v.n_new[b] = n;
  }
  if (b == 0) {
    v.counts[LIF_KV_CNT_FREE] = n_free - total;
    if (total) v.counts[KV_FREE_FROM] = page_list[total - 1] + 1;
    v.counts[LIF_KV_CNT_COPIES] = n_copies;
  }
  kv_plan(v, tokens + n, n);
}

// Table entries are handled in chunks of 32 of one row, a warp each.  The last row whose first chunk is
// <= chunk (rows without chunks have the next one's).
__device__ __forceinline__ int row_of_chunk(const int* first_chunk, int rows, int chunk) {
  int lo = 0, hi = rows;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first_chunk[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}
constexpr int kEarlyChunks = 4;              // a warp's chunks whose loads travel together and that stay in registers

// What fork and load have in common: new rows of the table from given ones, references counted anew.
// `from`: the rows' source, v.table (fork: row src[b]) or the caller's table (load: row b).
template <bool kSmall>
__global__ void __cluster_dims__(kSmall ? 1 : kKvCluster, 1, 1) __launch_bounds__(kKvPlanThreads)
kv_arrange_kernel(KvView v, const int32_t* from, const int32_t* src, const int32_t* len, const int32_t* n_new, int load) {
  extern __shared__ int held_by[];           // [n_pages] (small tables)
  __shared__ int s_src[kKvPlanThreads], s_pages[kKvPlanThreads], s_all[kKvPlanThreads], s_step[kKvPlanThreads],
      s_first[kKvPlanThreads];
  __shared__ int s_bad, s_free, s_lowest;
  constexpr int kParts = kSmall ? 1 : kKvCluster;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = kSmall ? 0 : (int)cluster.block_rank(), b = threadIdx.x, lane = b & 31;
  int* refs = kSmall ? held_by : v.page_tmp;
  const int per = (v.n_pages + kParts - 1) / kParts, p_lo = rank * per, p_hi = min(v.n_pages, p_lo + per);
  auto barrier = [&] {
    if (kSmall) __syncthreads(); else cluster.sync();
  };
  pdl_wait();
  // every CTA reads and judges all places
  const bool mine = b < v.max_seqs;
  int tokens = 0, news = 0, old = 0;
  bool bad = false;
  s_src[b] = b;
  if (mine) old = kv_pages_of(v.lens[b], v.page_shift);
  if (mine && load) {
    tokens = len[b];
    news = n_new ? n_new[b] : 0;
    bad = tokens < 0 || tokens > v.max_pages << v.page_shift || news < 0 || news > v.max_new || news > tokens;
  } else if (mine) {
    const int s = src ? src[b] : b;
    const int want = len ? len[b] : -1;
    bad = s < -1 || s >= v.max_seqs;
    const int held = bad || s < 0 ? 0 : v.lens[s];
    tokens = want == -1 || s < 0 ? held : want;
    bad = bad || tokens < 0 || tokens > held;
    s_src[b] = s < 0 ? 0 : s;
  }
  const int pages = bad ? 0 : kv_pages_of(tokens, v.page_shift);
  s_pages[b] = pages;
  s_all[b] = max(pages, old);
  s_step[b] = news > 0 ? (tokens - news) >> v.page_shift : 0x7fffffff;
  if (b == 0) s_bad = s_free = 0, s_lowest = v.n_pages;
  for (int p = p_lo + b; p < p_hi; p += kKvPlanThreads) refs[p] = 0;
  unsigned long long sums;
  s_first[b] = (int)block_scan((unsigned long long)((s_all[b] + 31) / 32) | (unsigned long long)bad << 40, &sums);
  const int chunks = (int)(sums & 0xffffffffffULL);
  if (sums >> 40) {                          // the same in every CTA
    if (rank == 0 && b == 0) kv_refuse(v, LIF_ERR_INVALID_ARG);
    return;
  }
  barrier();                                 // references are zero, lengths read, s_first written
  const int c0 = rank * (kKvPlanThreads / 32) + (b >> 5), step = kParts * (kKvPlanThreads / 32);
  auto entry = [&](int c, int* row, int* j) {
    *row = row_of_chunk(s_first, v.max_seqs, c);
    *j = (c - s_first[*row]) * 32 + lane;
    int page = -1;
    if (*j < s_pages[*row]) {
      page = from[(size_t)s_src[*row] * v.max_pages + *j];
      if (page < 0 || page >= v.n_pages) page = -2;
    }
    return page;
  };
  auto count = [&](int page) {
    if (page == -2) s_bad = 1;
    if (page >= 0) atomicAdd(refs + page, 1);
  };
  int row[kEarlyChunks], col[kEarlyChunks], early[kEarlyChunks];
#pragma unroll
  for (int i = 0; i < kEarlyChunks; ++i) {
    early[i] = -1;
    if (c0 + i * step < chunks) early[i] = entry(c0 + i * step, &row[i], &col[i]);
  }
#pragma unroll
  for (int i = 0; i < kEarlyChunks; ++i) count(early[i]);
  for (int c = c0 + kEarlyChunks * step; c < chunks; c += step) {
    int r, j;
    const int page = entry(c, &r, &j);
    if (j < s_pages[r]) v.table_tmp[(size_t)r * v.max_pages + j] = page;   // (-2 too: it is read again below)
    count(page);
  }
  barrier();                                 // references are counted
  if (load && n_new) {
    // pages that the step's tokens lie in belong to one entry only
    auto alone = [&](int page, int r, int j) {
      if (page >= 0 && j >= s_step[r] && (kSmall ? refs[page] : __ldcg(refs + page)) != 1) s_bad = 1;
    };
#pragma unroll
    for (int i = 0; i < kEarlyChunks; ++i)
      if (c0 + i * step < chunks) alone(early[i], row[i], col[i]);
    for (int c = c0 + kEarlyChunks * step; c < chunks; c += step) {
      const int r = row_of_chunk(s_first, v.max_seqs, c), j = (c - s_first[r]) * 32 + lane;
      if (j < s_pages[r]) alone(v.table_tmp[(size_t)r * v.max_pages + j], r, j);
    }
  }
  barrier();
  bool any = s_bad != 0;
  if (!kSmall)
    for (int c = 0; c < kKvCluster; ++c) any = any || *cluster.map_shared_rank(&s_bad, c) != 0;
  if (any) {                                 // the same in every CTA
    if (rank == 0 && b == 0) kv_refuse(v, LIF_ERR_INVALID_ARG);
    barrier();                               // nobody leaves while its flag may be read
    return;
  }
#pragma unroll
  for (int i = 0; i < kEarlyChunks; ++i)
    if (c0 + i * step < chunks && col[i] < s_all[row[i]]) v.table[(size_t)row[i] * v.max_pages + col[i]] = early[i];
  for (int c = c0 + kEarlyChunks * step; c < chunks; c += step) {
    const int r = row_of_chunk(s_first, v.max_seqs, c), j = (c - s_first[r]) * 32 + lane;
    if (j < s_all[r]) v.table[(size_t)r * v.max_pages + j] = j < s_pages[r] ? v.table_tmp[(size_t)r * v.max_pages + j] : -1;
  }
  int free_here = 0, lowest = v.n_pages;
  for (int p = p_lo + b; p < p_hi; p += kKvPlanThreads) {
    const int r = kSmall ? refs[p] : __ldcg(refs + p);
    v.refs[p] = r;
    if (r == 0) {
      ++free_here;
      lowest = min(lowest, p);
    }
  }
  free_here = __reduce_add_sync(~0u, free_here);
  lowest = __reduce_min_sync(~0u, lowest);
  if (lane == 0) {
    atomicAdd(&s_free, free_here);
    atomicMin(&s_lowest, lowest);
  }
  barrier();
  if (rank == 0) {
    if (b == 0) {
      int n = s_free, p = s_lowest;
      if (!kSmall)
        for (int c = 1; c < kKvCluster; ++c) {
          n += *cluster.map_shared_rank(&s_free, c);
          p = min(p, *cluster.map_shared_rank(&s_lowest, c));
        }
      v.counts[LIF_KV_CNT_FREE] = n;
      v.counts[KV_FREE_FROM] = p;
    }
    if (mine) {
      v.lens[b] = tokens;
      v.n_new[b] = news;
    }
    kv_plan(v, tokens, news);
  }
  if (!kSmall) cluster.sync();
}

// Tables that one CTA handles: refs and their ids in 16 bits in its shared memory.
constexpr int kSmallPages = 40000, kSmallTable = 1 << 16;

__global__ void __launch_bounds__(kKvPlanThreads)
kv_compact_small_kernel(KvView v) {
  extern __shared__ unsigned short ids[];    // [n_pages] new ids of those that move, [n_pages / 2] from, [n_pages / 2] to
  __shared__ int s_first[kKvPlanThreads], s_pages[kKvPlanThreads];
  __shared__ int s_moves;
  pdl_wait();
  const int b = threadIdx.x, lane = b & 31;
  unsigned short *from = ids + v.n_pages, *to = from + v.n_pages / 2;
  auto refs_of = [&](int p) {                // four pages' flags
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < v.n_pages && v.refs[p + i] > 0) mask |= 1u << i;
    return mask;
  };
  unsigned held = refs_of(4 * b);
  const int used = v.n_pages - v.counts[LIF_KV_CNT_FREE];
  s_pages[b] = b < v.max_seqs ? kv_pages_of(v.lens[b], v.page_shift) : 0;
  if (b == 0) s_moves = 0;
  unsigned long long chunks64;
  s_first[b] = (int)block_scan((s_pages[b] + 31) / 32, &chunks64);
  const int chunks = (int)chunks64;
  __syncthreads();
  // the table's entries travel while the lists are made
  const int c0 = b >> 5, step = kKvPlanThreads / 32;
  int32_t* at[kEarlyChunks];
  int early[kEarlyChunks];
  auto place = [&](int c) -> int32_t* {
    const int r = row_of_chunk(s_first, v.max_seqs, c), j = (c - s_first[r]) * 32 + lane;
    return j < s_pages[r] ? v.table + (size_t)r * v.max_pages + j : nullptr;
  };
#pragma unroll
  for (int i = 0; i < kEarlyChunks; ++i) {
    at[i] = c0 + i * step < chunks ? place(c0 + i * step) : nullptr;
    early[i] = at[i] ? *at[i] : 0;
  }
  // holes below `used`, ascending, and used pages from there on, descending: equally many
  int before = 0;
  for (int p0 = 0;;) {
    unsigned long long here;
    int below = before + (int)block_scan(__popc(held), &here), moves = 0;
    const int p = p0 + 4 * b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = held >> i & 1;
      if (p + i < v.n_pages) {
        if (!u && p + i < used) to[p + i - below] = (unsigned short)(p + i);
        if (u && p + i >= used) {
          from[used - 1 - below] = (unsigned short)(p + i);
          ++moves;
        }
      }
      below += u;
    }
    moves = __reduce_add_sync(~0u, moves);
    if (lane == 0 && moves) atomicAdd(&s_moves, moves);
    before += (int)here;
    p0 += 4 * kKvPlanThreads;
    if (p0 >= v.n_pages) break;
    held = refs_of(p0 + 4 * b);
  }
  __syncthreads();
  const int moves = s_moves;
  for (int j = b; j < moves; j += kKvPlanThreads) {
    const int s = from[j], d = to[j];
    ids[s] = (unsigned short)d;
    v.list_a[j] = s;
    v.list_b[j] = d;
    v.copy_tokens[j] = 1 << v.page_shift;
    v.refs[d] = v.refs[s];
    v.refs[s] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEarlyChunks; ++i)
    if (at[i] && early[i] >= used) *at[i] = ids[early[i]];
  for (int c = c0 + kEarlyChunks * step; c < chunks; c += step) {
    int32_t* e = place(c);
    if (e && *e >= used) *e = ids[*e];
  }
  if (b == 0) {
    v.counts[LIF_KV_CNT_COPIES] = moves;
    v.counts[KV_FREE_FROM] = used;
  }
}

__global__ void __cluster_dims__(kKvCluster, 1, 1) __launch_bounds__(kKvPlanThreads)
kv_compact_kernel(KvView v) {
  __shared__ int s_used, s_moves;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), tid = threadIdx.x;
  pdl_wait();
  if (tid == 0) s_used = s_moves = 0;
  __syncthreads();
  const int per = ((v.n_pages + kKvCluster - 1) / kKvCluster + 3) & ~3;
  const int p_lo = min(v.n_pages, rank * per), p_hi = min(v.n_pages, p_lo + per);
  int mine = 0;
  for (int p = p_lo + tid; p < p_hi; p += kKvPlanThreads) mine += v.refs[p] > 0;
  mine = __reduce_add_sync(~0u, mine);
  if ((tid & 31) == 0) atomicAdd(&s_used, mine);
  cluster.sync();
  int used = 0, before = 0;                  // in all; below this CTA's pages
  for (int c = 0; c < kKvCluster; ++c) {
    const int u = *cluster.map_shared_rank(&s_used, c);
    used += u;
    if (c < rank) before += u;
  }
  // holes below `used`, ascending, and used pages from there on, descending: equally many
  for (int p0 = p_lo; p0 < p_hi; p0 += 4 * kKvPlanThreads) {
    const int p = p0 + 4 * tid;
    int r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p + i < p_hi ? v.refs[p + i] > 0 : 0;
    unsigned long long here;
    int below = before + (int)block_scan(r[0] + r[1] + r[2] + r[3], &here);
    int moves = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + i < p_hi) {
        if (!r[i] && p + i < used) v.list_b[p + i - below] = p + i;
        if (r[i] && p + i >= used) {
          v.list_a[used - 1 - below] = p + i;
          ++moves;
        }
      }
      below += r[i];
    }
    moves = __reduce_add_sync(~0u, moves);
    if ((tid & 31) == 0) atomicAdd(&s_moves, moves);
    before += (int)here;
  }
  cluster.sync();
  int moves = 0;
  for (int c = 0; c < kKvCluster; ++c) moves += *cluster.map_shared_rank(&s_moves, c);
  for (int j = rank * kKvPlanThreads + tid; j < moves; j += kKvCluster * kKvPlanThreads) {
    const int s = __ldcg(v.list_a + j), d = __ldcg(v.list_b + j);
    v.page_tmp[s] = d;
    v.copy_tokens[j] = 1 << v.page_shift;
    v.refs[d] = v.refs[s];
    v.refs[s] = 0;
  }
  cluster.sync();
  for (int r = rank; r < v.max_seqs; r += kKvCluster) {
    const int n = kv_pages_of(v.lens[r], v.page_shift);
    for (int j = tid; j < n; j += kKvPlanThreads) {
      int32_t* e = v.table + (size_t)r * v.max_pages + j;
      if (*e >= used) *e = __ldcg(v.page_tmp + *e);
    }
  }
  if (rank == 0 && tid == 0) {
    v.counts[LIF_KV_CNT_COPIES] = moves;
    v.counts[KV_FREE_FROM] = used;
  }
  cluster.sync();                            // nobody leaves while its counts may be read
}

__global__ void __launch_bounds__(kKvPlanThreads) kv_reset_kernel(KvView v) {
  pdl_wait();
  const size_t at = (size_t)blockIdx.x * kKvPlanThreads + threadIdx.x, step = (size_t)gridDim.x * kKvPlanThreads;
  for (size_t i = at; i < (size_t)v.max_seqs * v.max_pages; i += step) v.table[i] = -1;
  for (size_t i = at; i < (size_t)v.n_pages; i += step) v.refs[i] = 0;
  if (at < (size_t)v.max_seqs) v.lens[at] = v.n_new[at] = 0;
  if (at < LIF_KV_CNT_LEN) v.counts[at] = at == LIF_KV_CNT_FREE ? v.n_pages : 0;
}

__global__ void kv_clear_kernel(KvView v) {
  pdl_wait();
  v.counts[LIF_KV_CNT_STATUS] = LIF_OK;
}

// Rows of pages list_a[i] to pages list_b[i], every layer and head.  Unit: 4 KB of one head's rows, a
// warp, eight 16-byte loads of a lane on their way together, the stores marked as not read again (82 MB of 16-row
// beams' pages: 33 us with the calls ahead of it, 37 without the mark; 0.55 GB: 182 us, 92% of measured HBM, with
// sixteen CTAs an SM to follow one another where four that stayed took 193).
constexpr int kCopyUnit = 4096;
__global__ void __launch_bounds__(kThreads)
kv_copy_pages_kernel(KvView v, uint4* pages, int n_layers, int head_bytes, int units_per_head) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long heads = 2 * v.n_kv_heads, per_copy = heads * n_layers * units_per_head;
  const long long n = per_copy * v.counts[LIF_KV_CNT_COPIES];
  const size_t page_vec = (size_t)heads * head_bytes / 16, layer_vec = page_vec * v.n_pages;
  const int row_bytes = head_bytes >> v.page_shift;
  for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < n;
       u += (long long)gridDim.x * (kThreads / 32)) {
    const int i = (int)(u / per_copy);
    const int in = (int)(u - i * per_copy), part = in % units_per_head, lh = in / units_per_head;
    const int bytes = min(kCopyUnit, v.copy_tokens[i] * row_bytes - part * kCopyUnit);
    if (bytes <= 0) continue;
    const size_t within = (size_t)(lh / (int)heads) * layer_vec +
                          ((size_t)(lh % (int)heads) * head_bytes + (size_t)part * kCopyUnit) / 16;
    const uint4* s = pages + within + (size_t)v.list_a[i] * page_vec;
    uint4* d = pages + within + (size_t)v.list_b[i] * page_vec;
    uint4 x[kCopyUnit / 512];
#pragma unroll
    for (int k = 0; k < kCopyUnit / 512; ++k)
      if ((k * 32 + lane) * 16 < bytes) x[k] = ld_stream16(s + k * 32 + lane);
#pragma unroll
    for (int k = 0; k < kCopyUnit / 512; ++k)
      if ((k * 32 + lane) * 16 < bytes) __stcs(d + k * 32 + lane, x[k]);
  }
}

bool small_tables(const KvView& v) { return v.n_pages <= kSmallPages && (long long)v.max_seqs * v.max_pages <= kSmallTable; }

cudaError_t launch_arrange(const lif_kv* kv, const int32_t* from, const int32_t* src, const int32_t* len, const int32_t* n_new,
                           int load, cudaStream_t st) {
  if (small_tables(kv->v))
    return launch_k(kv_arrange_kernel<true>, dim3(1), dim3(kKvPlanThreads), (size_t)kv->v.n_pages * 4, st, 1, kv->v, from, src, len,
                    n_new, load);
  return launch_k(kv_arrange_kernel<false>, dim3(kKvCluster), dim3(kKvPlanThreads), 0, st, 1, kv->v, from, src, len, n_new, load);
}

cudaError_t launch_copies(const lif_kv* kv, cudaStream_t st) {
  const lif_kv_desc& d = kv->desc;
  const int head_bytes = d.page_tokens * d.head_dim * 2;
  return launch_k(kv_copy_pages_kernel, dim3(kv->n_sm * 16), dim3(kThreads), 0, st, 1, kv->v, (uint4*)d.dev_pages,
                  d.n_layers, head_bytes, (head_bytes + kCopyUnit - 1) / kCopyUnit);
}

// ---- host side -------------------------------------------------------------------------------------

bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

lif_status check_desc(const lif_kv_desc* d) {
  if (!d) return LIF_ERR_INVALID_ARG;
  const int D = d->head_dim;
  if (D != 64 && D != 80 && D != 96 && D != 128 && D != 256) return LIF_ERR_INVALID_ARG;
  if (d->n_layers < 1 || d->n_layers > 1024) return LIF_ERR_INVALID_ARG;
  if (d->n_kv_heads < 1 || d->n_heads < 1 || d->n_heads > 1024 || d->n_heads % d->n_kv_heads) return LIF_ERR_INVALID_ARG;
  if (d->dtype != LIF_TYPE_F16 && d->dtype != LIF_TYPE_BF16) return LIF_ERR_INVALID_ARG;
  if (!is_pow2(d->page_tokens) || d->page_tokens < 8 || d->page_tokens > 256) return LIF_ERR_INVALID_ARG;
  if (d->n_pages < 1 || d->n_pages > 1 << 24) return LIF_ERR_INVALID_ARG;
  if (d->max_seqs < 1 || d->max_seqs > LIF_KV_MAX_SEQS) return LIF_ERR_INVALID_ARG;
  if (d->max_pages < 1 || (long long)d->max_pages * d->page_tokens > 1 << 30) return LIF_ERR_INVALID_ARG;
  if (d->max_new < 1 || d->max_new > LIF_KV_MAX_NEW) return LIF_ERR_INVALID_ARG;
  if (d->window < 0 || d->window > 1 << 30) return LIF_ERR_INVALID_ARG;
  if (!(d->scale >= 0.f) || !isfinite(d->scale)) return LIF_ERR_INVALID_ARG;
  if (d->norm < LIF_NORM_NONE || d->norm > LIF_NORM_LAYER) return LIF_ERR_INVALID_ARG;
  if (d->norm != LIF_NORM_NONE && (!(d->norm_eps >= 0.f) || !isfinite(d->norm_eps))) return LIF_ERR_INVALID_ARG;
  if (d->rope < LIF_ROPE_NONE || d->rope > LIF_ROPE_INTERLEAVED) return LIF_ERR_INVALID_ARG;
  if (d->rope == LIF_ROPE_NONE ? d->rope_dims != 0 : (d->rope_dims < 2 || d->rope_dims > D || d->rope_dims % 2))
    return LIF_ERR_INVALID_ARG;
  if (d->rope != LIF_ROPE_NONE && !isfinite(d->rope_scale)) return LIF_ERR_INVALID_ARG;
  // Tiles are numbered in 32 bits.  Sums of a tile's number and a share of them (of 32 shares at least) stay below
  // 2^31 too: kv_plan and the attention kernels' walk form them.
  constexpr long long kMaxTiles = (1LL << 31) - (1LL << 26);
  const long long rows = (long long)(d->n_heads / d->n_kv_heads) * d->max_new;
  const long long per_block = 16 * kv_row_tiles(*d), blocks = (rows + per_block - 1) / per_block;
  const long long tiles = ((long long)d->max_pages * d->page_tokens + kKvTile - 1) / kKvTile;
  if (tiles * d->max_seqs > kMaxTiles / (d->n_kv_heads * blocks)) return LIF_ERR_INVALID_ARG;
  return LIF_OK;
}

KvWorkspace plan(const lif_kv_desc& d) {
  KvWorkspace w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) / 256 * 256;
    return at;
  };
  const size_t table = (size_t)d.max_seqs * d.max_pages * 4, pages = (size_t)d.n_pages * 4;
  w.counts = take(LIF_KV_CNT_LEN * 4);
  w.lens = take((size_t)d.max_seqs * 4);
  w.n_new = take((size_t)d.max_seqs * 4);
  w.table = take(table);
  w.table_tmp = take(table);
  w.refs = take(pages);
  w.page_tmp = take(pages);
  w.list_a = take(pages);
  w.list_b = take(pages);
  w.copy_tokens = take(pages);
  w.seq_plan = take((size_t)d.max_seqs * 16);
  w.run_plan = take((size_t)(kKvMaxCtas + kv_max_runs(d)) * 16);
  w.joins = take((size_t)kv_max_runs(d) * 16);
  w.turns = take((size_t)d.rope_dims / 2 * 8);
  w.partials = take((size_t)2 * kv_max_runs(d) * kv_slot_rows(d) * (d.head_dim + 4) * 4);
  w.total = off;
  return w;
}

// 2^64ths of a turn: position * this, modulo 2^64, is the angle at any position without a rounding
// that grows with it (2^-65 turns per position, below 2^-34 of a turn at position 2^30).
uint64_t turn_fraction(double radians) {
  long double t = (long double)radians / 6.283185307179586476925286766559L;
  t -= roundl(t);
  const long double s = roundl(t * 18446744073709551616.0L);
  return s >= 9223372036854775808.0L ? (uint64_t)1 << 63 : (uint64_t)(int64_t)s;
}

// [max_seqs][max_new][n_heads][head_dim]
size_t query_bytes(const lif_kv_desc& d) { return (size_t)d.max_seqs * d.max_new * d.n_heads * d.head_dim * 2; }

// Does any row of an operand of append lie in the packed block of queries at `out`?
bool touches(const lif_kv_rows& r, int heads, const lif_kv_desc& d, const void* out) {
  const long long tokens = (long long)d.max_seqs * d.max_new, row = d.head_dim * 2;
  const long long token = r.token_stride * 2, head = r.head_stride * 2, n = (long long)query_bytes(d);
  const long long at = (long long)((uintptr_t)r.dev - (uintptr_t)out);          // of the block's first byte
  if (at >= n || at + (tokens - 1) * token + (heads - 1) * head + row <= 0) return false;
  for (int h = 0; h < heads; ++h) {
    const long long b = at + h * head;               // this head's rows begin at b + t * token
    const long long t = b + row > 0 ? 0 : token ? (-b - row) / token + 1 : tokens;   // the first that ends inside or behind
    if (t < tokens && b + t * token < n) return true;
  }
  return false;
}

lif_status enter(const lif_kv* kv) {
  if (!kv) return LIF_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return LIF_ERR_CUDA;
  }
  return dev == kv->device ? LIF_OK : LIF_ERR_STATE;
}

lif_status done(cudaError_t e) {
  if (e == cudaSuccess) return LIF_OK;
  cudaGetLastError();
  return LIF_ERR_CUDA;
}

}  // namespace
}  // namespace lif

using namespace lif;

extern "C" {

lif_status lif_kv_workspace_bytes(const lif_kv_desc* desc, size_t* out_bytes) {
  if (!out_bytes) return LIF_ERR_INVALID_ARG;
  const lif_status s = check_desc(desc);
  if (s != LIF_OK) return s;
  *out_bytes = plan(*desc).total;
  return LIF_OK;
}

lif_status lif_kv_create(const lif_kv_desc* desc, lif_kv** out) {
  if (!out) return LIF_ERR_INVALID_ARG;
  *out = nullptr;
  const lif_status s = check_desc(desc);
  if (s != LIF_OK) return s;
  if (!desc->dev_pages || !desc->dev_workspace) return LIF_ERR_INVALID_ARG;
  const int pairs = desc->rope_dims / 2;
  if (pairs && !desc->host_rope_freq) return LIF_ERR_INVALID_ARG;
  uint64_t turns[128];
  for (int i = 0; i < pairs; ++i) {
    const double f = desc->host_rope_freq[i];
    if (!(fabs(f) <= 6.2831853071795865)) return LIF_ERR_INVALID_ARG;
    turns[i] = turn_fraction(f);
  }
  if (!aligned(desc->dev_pages, 16) || !aligned(desc->dev_workspace, 256)) return LIF_ERR_ALIGNMENT;
  const KvWorkspace w = plan(*desc);
  if (desc->workspace_bytes < w.total) return LIF_ERR_INVALID_ARG;

  lif_kv* kv = new (std::nothrow) lif_kv();
  if (!kv) return LIF_ERR_STATE;
  kv->desc = *desc;
  kv->desc.host_rope_freq = nullptr;         // not the library's to keep
  kv->row_tiles = kv_row_tiles(*desc);
  kv->scale = desc->scale > 0.f ? desc->scale : 1.f / sqrtf((float)desc->head_dim);
  unsigned char* base = (unsigned char*)desc->dev_workspace;
  KvView& v = kv->v;
  v.counts = (int32_t*)(base + w.counts);
  v.lens = (int32_t*)(base + w.lens);
  v.n_new = (int32_t*)(base + w.n_new);
  v.table = (int32_t*)(base + w.table);
  v.table_tmp = (int32_t*)(base + w.table_tmp);
  v.refs = (int32_t*)(base + w.refs);
  v.page_tmp = (int32_t*)(base + w.page_tmp);
  v.list_a = (int32_t*)(base + w.list_a);
  v.list_b = (int32_t*)(base + w.list_b);
  v.copy_tokens = (int32_t*)(base + w.copy_tokens);
  v.seq_plan = (int4*)(base + w.seq_plan);
  v.run_plan = (int4*)(base + w.run_plan);
  v.joins = (int4*)(base + w.joins);
  v.turns = (const uint64_t*)(base + w.turns);
  v.partials = (float*)(base + w.partials);
  v.max_seqs = desc->max_seqs;
  v.max_pages = desc->max_pages;
  v.n_pages = desc->n_pages;
  v.max_new = desc->max_new;
  v.page_shift = 0;
  while (1 << v.page_shift < desc->page_tokens) ++v.page_shift;
  v.window = desc->window;
  v.n_heads = desc->n_heads;
  v.n_kv_heads = desc->n_kv_heads;
  v.group = desc->n_heads / desc->n_kv_heads;
  v.head_dim = desc->head_dim;
  v.rows_per_block = 16 * kv->row_tiles;
  v.max_runs = kv_max_runs(*desc);
  v.slot_rows = kv_slot_rows(*desc);
  v.slot_floats = v.slot_rows * (desc->head_dim + 4);

  int per_sm = 0;
  bool ok = cudaGetDevice(&kv->device) == cudaSuccess &&
            cudaDeviceGetAttribute(&kv->n_sm, cudaDevAttrMultiProcessorCount, kv->device) == cudaSuccess &&
            kv_attention_configure(kv, &per_sm) && per_sm > 0 && kv->n_sm * per_sm >= 32;   // (kMaxTiles)
  v.ctas = ok ? kv->n_sm * per_sm < kKvMaxCtas ? kv->n_sm * per_sm : kKvMaxCtas : 0;
  ok = ok && cudaFuncSetAttribute(kv_reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kReserveListMost * 4) == cudaSuccess &&
       cudaFuncSetAttribute(kv_arrange_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallPages * 4) == cudaSuccess &&
       cudaFuncSetAttribute(kv_compact_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallPages * 4 + 4) == cudaSuccess;
  ok = ok && (pairs == 0 || cudaMemcpy(base + w.turns, turns, (size_t)pairs * 8, cudaMemcpyHostToDevice) == cudaSuccess);
  ok = ok && lif_kv_reset(kv, nullptr) == LIF_OK && cudaDeviceSynchronize() == cudaSuccess;
  if (!ok) {
    cudaGetLastError();
    delete kv;
    return LIF_ERR_CUDA;
  }
  *out = kv;
  return LIF_OK;
}

lif_status lif_kv_destroy(lif_kv* kv) {
  if (!kv) return LIF_ERR_INVALID_ARG;
  delete kv;
  return LIF_OK;
}

lif_status lif_kv_get_state(lif_kv* kv, lif_kv_state* host_out) {
  if (!kv || !host_out) return LIF_ERR_INVALID_ARG;
  *host_out = lif_kv_state{kv->v.counts, kv->v.lens, kv->v.n_new, kv->v.table, kv->v.refs};
  return LIF_OK;
}

lif_status lif_kv_reset(lif_kv* kv, void* stream) {
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_k(kv_reset_kernel, dim3(kv->n_sm), dim3(kKvPlanThreads), 0, (cudaStream_t)stream, 1, kv->v));
}

lif_status lif_kv_reserve(lif_kv* kv, const int32_t* dev_n_new, void* stream) {
  if (!kv || !dev_n_new) return LIF_ERR_INVALID_ARG;
  if (!aligned(dev_n_new, 4)) return LIF_ERR_ALIGNMENT;
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = launch_k(kv_reserve_kernel, dim3(1), dim3(kKvPlanThreads), (size_t)reserve_list(kv->v) * 4, st, 1, kv->v, dev_n_new);
  if (e == cudaSuccess) e = launch_copies(kv, st);
  return done(e);
}

lif_status lif_kv_fork(lif_kv* kv, const int32_t* dev_src, const int32_t* dev_len, void* stream) {
  if (!kv) return LIF_ERR_INVALID_ARG;
  if (!aligned(dev_src, 4) || !aligned(dev_len, 4)) return LIF_ERR_ALIGNMENT;
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_arrange(kv, kv->v.table, dev_src, dev_len, nullptr, 0, (cudaStream_t)stream));
}

lif_status lif_kv_load(lif_kv* kv, const int32_t* dev_lens, const int32_t* dev_table, const int32_t* dev_n_new,
                       void* stream) {
  if (!kv || !dev_lens || !dev_table) return LIF_ERR_INVALID_ARG;
  if (!aligned(dev_lens, 4) || !aligned(dev_table, 4) || !aligned(dev_n_new, 4)) return LIF_ERR_ALIGNMENT;
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_arrange(kv, dev_table, nullptr, dev_lens, dev_n_new, 1, (cudaStream_t)stream));
}

lif_status lif_kv_compact(lif_kv* kv, void* stream) {
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = small_tables(kv->v)
                      ? launch_k(kv_compact_small_kernel, dim3(1), dim3(kKvPlanThreads), (size_t)kv->v.n_pages * 4 + 4, st, 1, kv->v)
                      : launch_k(kv_compact_kernel, dim3(kKvCluster), dim3(kKvPlanThreads), 0, st, 1, kv->v);
  if (e == cudaSuccess) e = launch_copies(kv, st);
  return done(e);
}

lif_status lif_kv_append(lif_kv* kv, int32_t layer, const lif_kv_rows* q, const lif_kv_rows* k, const lif_kv_rows* v,
                         const lif_kv_norms* norms, void* dev_q_out, void* stream) {
  if (!kv || !q || !k || !v || !dev_q_out || layer < 0 || layer >= kv->desc.n_layers) return LIF_ERR_INVALID_ARG;
  for (const lif_kv_rows* r : {q, k, v}) {
    if (!r->dev || r->token_stride < 0 || r->head_stride < 0) return LIF_ERR_INVALID_ARG;
    if (!aligned(r->dev, 16) || r->token_stride % 8 || r->head_stride % 8) return LIF_ERR_ALIGNMENT;
  }
  if (!aligned(dev_q_out, 16)) return LIF_ERR_ALIGNMENT;
  const lif_kv_desc& d = kv->desc;
  const bool in_place = q->dev == dev_q_out && (d.n_heads == 1 || q->head_stride == d.head_dim) &&
                        (d.max_seqs * d.max_new == 1 || q->token_stride == (int64_t)d.n_heads * d.head_dim);
  if ((!in_place && touches(*q, d.n_heads, d, dev_q_out)) || touches(*k, d.n_kv_heads, d, dev_q_out) ||
      touches(*v, d.n_kv_heads, d, dev_q_out))
    return LIF_ERR_INVALID_ARG;
  lif_kv_norms n = {};
  if (kv->desc.norm != LIF_NORM_NONE) {
    if (!norms || !norms->dev_q_weight || !norms->dev_k_weight) return LIF_ERR_INVALID_ARG;
    n = *norms;
    if (kv->desc.norm == LIF_NORM_RMS) n.dev_q_bias = n.dev_k_bias = nullptr;
    if (!aligned(n.dev_q_weight, 16) || !aligned(n.dev_k_weight, 16) || !aligned(n.dev_q_bias, 16) ||
        !aligned(n.dev_k_bias, 16))
      return LIF_ERR_ALIGNMENT;
  }
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_kv_append(kv, layer, *q, *k, *v, n, dev_q_out, (cudaStream_t)stream));
}

lif_status lif_kv_attention(lif_kv* kv, int32_t layer, const void* dev_q, void* dev_out, void* stream) {
  if (!kv || !dev_q || !dev_out || layer < 0 || layer >= kv->desc.n_layers) return LIF_ERR_INVALID_ARG;
  if (!aligned(dev_q, 16) || !aligned(dev_out, 16)) return LIF_ERR_ALIGNMENT;
  // A row of queries is read again by every CTA that has a piece of it, after others have written theirs.
  const uintptr_t from = (uintptr_t)dev_q, to = (uintptr_t)dev_out;
  if ((from < to ? to - from : from - to) < query_bytes(kv->desc)) return LIF_ERR_INVALID_ARG;
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_kv_attention(kv, layer, dev_q, dev_out, (cudaStream_t)stream));
}

lif_status lif_kv_get_stats(lif_kv* kv, int32_t* host_counts) {
  if (!kv || !host_counts) return LIF_ERR_INVALID_ARG;
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(host_counts, kv->v.counts, LIF_KV_CNT_LEN * 4, cudaMemcpyDeviceToHost);
  return done(e);
}

lif_status lif_kv_clear_status(lif_kv* kv, void* stream) {
  const lif_status s = enter(kv);
  if (s != LIF_OK) return s;
  return done(launch_k(kv_clear_kernel, dim3(1), dim3(1), 0, (cudaStream_t)stream, 1, kv->v));
}

}  // extern "C"
