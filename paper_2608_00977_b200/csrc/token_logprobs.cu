// Log probabilities of given columns, entropy, rank and the best columns of rows of scores, and the backward
// pass of the log probability and the entropy.
//
// With z_v = scale x_v over the columns v of a row:
//   logprob = z_y - log sum_v e^{z_v},   H = -sum_v p_v log p_v,   rank = #{x_v > x_y} + #{x_v = x_y, v < y},
//   top k   = the k columns first in the order (x descending, v ascending)
//   d x_v   = scale (g ([v = y] - p_v) - h p_v (log p_v + H)),  g, h = gradients of logprob and H.
//
// Forward: one pass over the row.  A thread keeps the running maximum, sum and entropy sum of its own blocks
// (every NT-th pair of 16-byte chunks of the CTA's part of the row); the parts are joined thread -> warp -> CTA ->
// cluster in a fixed order.  The running maximum is also what finds the best columns: the K-th largest of the
// threads' maxima is a lower bound of the K-th largest element, and only the K threads (and a few more, the bound
// comes from a histogram) whose maximum reaches it can own one of the K best.  Each thread has also noted the
// maximum of every pair, so of those threads only the pairs that reach the bound are read again, little more than K
// of them, and their elements at or above the bound are ranked by counting.  All comparisons are on (value, index)
// pairs, which are distinct, so ties need no special case and constant rows cost no more than others.
//
// What bounds it (one B200, 6.55 TB/s copy rate; times are of the kernel alone, a call in a sequence of calls takes 2 to 7 us
// more).  Per element one 2^x (the unit gives 16 per clock and SM) and about 8 other instructions, with lists and rank about
// 11, with fp32 scores 21.  Many rows without lists come near the copy rate: 2048 x 100,000 bf16 76 us (62.6 for its bytes),
// 4096 x 20,000 fp32 55 us (50.1); with rank 62, with 10 best 68, with both 76 us, where issue slots are 66 % busy and a row's end
// takes a quarter of its time.  Few long rows fill no unit (64 x 1,000,000 bf16 with rank and 50 best: 47 us against 19.6 for its
// bytes, issue slots 58 % busy, the 2^x unit 36 %, memory 40 %): the statistics alone take 32 us, the rank and the list 7 to 8
// us each, and the time goes in steps by how clusters fit on the chip (47 us for 37 rows of 12 CTAs and for 64 of 6, 66 us
// for 74 of 6).
// One row is latency: 100,000 columns with 20 best 11.7 us, of which the pass takes 5.
#include <cooperative_groups.h>

#include <type_traits>

#include "rows.cuh"

namespace cg = cooperative_groups;

namespace tsid {
namespace {

constexpr int kCand = 1024;    // candidate elements
constexpr int kLists = 1024;   // places of all lists of a cluster
constexpr int kSel = 1024;     // selected entries of the table of maxima
constexpr int kNote = 32;      // entries per thread of that table

struct LpArgs {
  const void *x;
  int64_t stride;
  const void *y;   // targets or null
  int32_t y64, V, k;
  float scale;
  float *logprob, *entropy, *row_max, *log_sum;
  int32_t *rank;
  float *top_lp;
  int32_t *top_id;
};

__device__ __forceinline__ int64_t load_id(const void *ids, int64_t t, int is64) {
  return is64 ? static_cast<const int64_t *>(ids)[t] : (int64_t)static_cast<const int32_t *>(ids)[t];
}

// Elements of a block that lie above a threshold, as two sums.  thr is in the element's own type for 16-bit
// elements: a packed comparison gives 1.0 or 0.0 per element, and sums of up to 8 of them are exact.
template <typename T>
__device__ __forceinline__ f32x2 count_above(const uint32_t (&w)[8], const float *x, float thr) {
  if constexpr (sizeof(T) == 4) {
    f32x2 s = mk2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float a, b;
      asm("set.gt.f32.f32 %0, %1, %2;" : "=f"(a) : "f"(x[i]), "f"(thr));
      asm("set.gt.f32.f32 %0, %1, %2;" : "=f"(b) : "f"(x[i + 1]), "f"(thr));
      s = add2(s, mk2(a, b));
    }
    return s;
  } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162 t = __float2bfloat162_rn(thr);
    __nv_bfloat162 s = __hgt2(*reinterpret_cast<const __nv_bfloat162 *>(&w[0]), t);
#pragma unroll
    for (int i = 1; i < 8; ++i) s = __hadd2(s, __hgt2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]), t));
    return mk2(__low2float(s), __high2float(s));
  } else {
    const __half2 t = __float2half2_rn(thr);
    __half2 s = __hgt2(*reinterpret_cast<const __half2 *>(&w[0]), t);
#pragma unroll
    for (int i = 1; i < 8; ++i) s = __hadd2(s, __hgt2(*reinterpret_cast<const __half2 *>(&w[i]), t));
    return mk2(__low2float(s), __high2float(s));
  }
}
// the largest value of the element type below x (x finite or +inf, above the type's minus infinity)
template <typename T>
__device__ __forceinline__ float next_below(float x) {
  if constexpr (sizeof(T) == 4) {
    const uint32_t o = order_of(x) - 1u;
    return order_inv(o == 0x7fffffffu ? o - 1u : o);   // 0x7fffffff is minus zero, equal to zero
  } else {
    const T e = El<T>::from(x + 0.0f);
    const uint16_t b = *reinterpret_cast<const uint16_t *>(&e);
    const uint16_t p = b == 0 ? 0x8001 : (b & 0x8000) ? b + 1 : b - 1;
    return El<T>::load(reinterpret_cast<const T *>(&p));
  }
}

// Counting is quadratic: a list longer than this is first narrowed down to little more than k.
constexpr int kCount = 256;
// Keys of src (distinct, 0 = none, n slots with at least k keys) that reach a lower bound of the k-th largest, into
// dst; returns how many.  All threads call it; src and dst may be the same.
template <int NT>
__device__ __forceinline__ int narrow(const uint64_t *src, int n, uint64_t *dst, int k, KeyHist &hist, uint32_t *sh_lo,
                                      uint32_t *sh_hi, int32_t &count) {
  constexpr int NK = (kCand > kLists ? kCand : kLists) / NT, NW = NT / 32;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  uint64_t mine[NK];
  uint32_t top = 0, low = 0xffffffffu;
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    mine[i] = i * NT + tid < n ? src[i * NT + tid] : 0ull;
    if (mine[i]) {
      top = max(top, (uint32_t)(mine[i] >> 32));
      low = min(low, (uint32_t)(mine[i] >> 32));
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  low = __reduce_min_sync(0xffffffffu, low);
  __syncthreads();
  if (lane == 0) {
    sh_hi[w] = top;
    sh_lo[w] = low;
  }
  if (tid == 0) count = 0;
  __syncthreads();
  const uint64_t h64 = (uint64_t)__reduce_max_sync(0xffffffffu, lane < NW ? sh_hi[lane] : 0u) << 32 | 0xffffffffull;
  const uint64_t l64 = (uint64_t)__reduce_min_sync(0xffffffffu, lane < NW ? sh_lo[lane] : 0xffffffffu) << 32;
  const uint64_t L = kth_bound<NT, NK>(mine, l64, h64, k, k + max(k / 4, 8), hist);
#pragma unroll
  for (int i = 0; i < NK; ++i)
    if (mine[i] >= L && mine[i]) dst[atomicAdd(&count, 1)] = mine[i];
  __syncthreads();
  return count;
}
// keys of a list (padded with zeros to a multiple of 2) above one of them
__device__ __forceinline__ int count_larger(const uint64_t *list, int n, uint64_t mine) {
  int rk = 0;
#pragma unroll 4
  for (int j = 0; j < n; j += 2) {
    const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(&list[j]);
    rk += (o.x > mine) + (o.y > mine);
  }
  return rk;
}

template <typename T, int NT, bool RANK>
__global__ void __launch_bounds__(NT, 896 / NT) token_logprobs_kernel(const LpArgs a) {
  constexpr int n = 2 * El<T>::kPer16;   // elements of a pair
  constexpr int NW = NT / 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int64_t t = (int64_t)blockIdx.x / S;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;

  __shared__ Soft sh_soft[NW];
  __shared__ float sh_cnt[NW];
  __shared__ uint32_t sh_lo[NW], sh_hi[NW];
  __shared__ uint32_t note[kNote / 2][NT];   // upper 16 bits of the maxima of a thread's pairs (of 2^ng pairs each)
  __shared__ int32_t nsel, ncand;
  __shared__ KeyHist hist;
  // the lists take the ring's place when the pass is over
  __shared__ union Mem {
    PairRing<NT> ring;
    struct {
      uint64_t cand[kCand + 4];
      uint64_t lists[kLists + 2];   // [S][k], each in order, 0 = none; written by all CTAs of the cluster
      int32_t sel[kSel];
    } top;
  } sm;
  uint64_t *const cand = sm.top.cand, *const lists = sm.top.lists;
  int32_t *const sel = sm.top.sel;
  // written by the other CTAs of the cluster into its first CTA
  __shared__ Soft all_soft[kRowClusterMax];
  __shared__ int32_t all_cnt[kRowClusterMax];

  const RowChunks<T> r(static_cast<const T *>(a.x) + t * a.stride, a.V);
  const int32_t per = ((r.pairs >> 5) + S - 1) / S * 32;   // pairs of a CTA: whole groups of 32
  const int32_t p0 = min(part * per, r.pairs), p1 = min(p0 + per, r.pairs);
  PairStream<T, NT> stream(r, sm.ring, p0 + tid, p1);

  const float c = a.scale * kLog2e;
  // the target's own score; rank: an element of an earlier block is ahead when it is >= xt, i.e. above the next
  // value below xt, one of a later block when it is above xt
  int64_t y = -1;
  float xt = 0.f, before = 0.f;
  int32_t ygroup = -1;   // the target's group of 32 pairs
  bool count = false;
  if (a.y) {
    y = load_id(a.y, t, a.y64);
    if (y >= 0 && y < a.V) {
      xt = El<T>::load(r.row + y);
      if (RANK) {
        count = xt > -INFINITY;
        if (count) before = next_below<T>(xt);
        ygroup = (int32_t)((y + r.lead) / (32 * n));
      }
    }
  }

  // ---- the pass
  float mk = -INFINITY;     // maximum of this thread's elements, and the first chunk that holds it
  int32_t mchunk = 0;
  RunningSoft<n, true> sums(a.scale);
  f32x2 ahead2 = mk2(0.f, 0.f);
  const int k = a.k;
  const int iters = (p1 - p0 + NT - 1) / NT;
  int ng = 0, it = 0;
  while (iters > kNote << ng) ++ng;
  float noted = -INFINITY;
  auto take = [&](int32_t p, const uint32_t(&words)[8]) {
    float x[n];
    unpack<T, 8>(words, x);
    const float ca = chunk_max<T>(words[0], words[1], words[2], words[3]);
    const float cb = chunk_max<T>(words[4], words[5], words[6], words[7]);
    const float cm = fmaxf(ca, cb);
    if (k > 0) {
      noted = it & ((1 << ng) - 1) ? fmaxf(noted, cm) : cm;
      // toward zero, which keeps the order; entry e is half e & 1 of word e >> 1
      reinterpret_cast<uint16_t *>(&note[it >> (ng + 1)][tid])[(it >> ng) & 1] = (uint16_t)(__float_as_uint(noted) >> 16);
      ++it;
    }
    if (cm > mk) {
      mk = cm;
      mchunk = r.chunk(p) + (ca == cm ? 0 : 32);
    }
    sums.take(x, cm);
    if (RANK && count) {
      if (p >> 5 == ygroup) {
        const PairColumns<T> col(r, p);
        float more = 0.f;
#pragma unroll
        for (int i = 0; i < n; ++i) more += x[i] > xt || (x[i] == xt && col.at(i) < y) ? 1.f : 0.f;
        ahead2 = add2(ahead2, mk2(more, 0.f));
      } else {
        ahead2 = add2(ahead2, count_above<T>(words, x, p >> 5 < ygroup ? before : xt));
      }
    }
  };
  stream.run(take);

  // ---- join: thread -> warp -> CTA
  Soft v = sums.result(mk);
  float ahead = 0.f;   // up to 2^31 columns: a thread's count is exact in fp32, the joins add whole numbers
  if (RANK) {
    float a_0, a_1;
    un2(ahead2, a_0, a_1);
    ahead = a_0 + a_1;
  }
  v = soft_warp(v, c);
  const int32_t ahead_w = RANK ? __reduce_add_sync(0xffffffffu, (int32_t)ahead) : 0;
  if (S > 1) cluster.barrier_arrive();   // (1) past the pass: the first CTA's lists may be written
  const bool has = mk > -INFINITY;
  const uint32_t mo = order_of(mk) >> El<T>::kShift;
  const uint32_t whi = __reduce_max_sync(0xffffffffu, has ? mo : 0u);
  const uint32_t wlo = __reduce_min_sync(0xffffffffu, has ? mo : 0xffffffffu);
  if (lane == 0) {
    sh_soft[w] = v;
    sh_hi[w] = whi;
    sh_lo[w] = wlo;
    if (RANK) sh_cnt[w] = __int_as_float(ahead_w);
  }
  if (tid == 0) nsel = ncand = 0;
  if (S > 1) cluster.barrier_wait();     // (1)
  const int nhas = __syncthreads_count(has);
  if (w == 0) {
    Soft q;
    q.m = kLowest;
    q.s = q.u = 0.f;
    if (lane < NW) q = sh_soft[lane];
    q = soft_warp(q, c);
    int32_t cn = RANK && lane < NW ? __float_as_int(sh_cnt[lane]) : 0;
    cn = __reduce_add_sync(0xffffffffu, cn);
    if (lane == 0) {
      *(S > 1 ? cluster.map_shared_rank(&all_soft[part], 0) : &all_soft[0]) = q;
      *(S > 1 ? cluster.map_shared_rank(&all_cnt[part], 0) : &all_cnt[0]) = cn;
    }
  }

  // ---- this CTA's best k
  int nc = 0;
  if (k > 0) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, lane < NW ? sh_hi[lane] : 0u);
    const uint32_t lo = __reduce_min_sync(0xffffffffu, lane < NW ? sh_lo[lane] : 0xffffffffu);
    const int32_t nch = 2 * per, ch0 = 2 * p0;   // this CTA's chunks
    const int ib = 32 - __clz(nch);              // bits of a chunk's place among them
    const uint64_t key[1] = {has ? ((uint64_t)mo << ib | (uint32_t)(nch - 1 - (mchunk - ch0))) : 0ull};
    // smallest element key that is collected, (value order << 32) | ~index, and smallest thread key
    uint64_t floor_key = ((uint64_t)order_of(-INFINITY) << 32) + 0x100000000ull;   // every finite element
    if (nhas > k) {
      const uint64_t L = kth_bound<NT, 1>(key, (uint64_t)lo << ib, (((uint64_t)hi + 1) << ib) - 1, k, k + max(k / 2, 8), hist);
      // as an element key: value order, and the last element of the bound's chunk
      const uint32_t vo = (uint32_t)(L >> ib);
      const int32_t ch = max(ch0 + nch - 1 - (int32_t)(L & ((1ull << ib) - 1)), ch0);
      // the value's dropped low bits are all ones or all zeros for every element, so comparing the kept
      // bits is comparing the values
      floor_key = ((uint64_t)vo << (32 + El<T>::kShift)) | (uint32_t)~(uint32_t)(r.first(ch + 1) - 1);
      if (El<T>::kShift > 0 && !(vo >> (31 - El<T>::kShift)))   // negative: low order bits are ones
        floor_key |= (uint64_t)((1u << El<T>::kShift) - 1u) << 32;
    }
    // the elements of pair p at or above a key: found first, then one reservation for all of them
    auto offer = [&](int32_t p, const uint32_t(&words)[8], uint64_t least) {
      float x[n];
      unpack<T, 8>(words, x);
      if ((uint32_t)(least >> 32) == 0x7fffffffu) least = 0x8000000000000000ull;   // minus zero is zero
      const float low = order_inv((uint32_t)(least >> 32));
      const PairColumns<T> col(r, p);
      uint32_t hit = 0, tie = 0;
#pragma unroll
      for (int j = 0; j < n; ++j) {
        hit |= x[j] > low ? 1u << j : 0u;
        tie |= x[j] == low ? 1u << j : 0u;
      }
      if (tie) {   // of equal values the columns up to the key's
        const int64_t last = (int64_t)(uint32_t)~(uint32_t)least;
        const int na = (int)max((int64_t)0, min((int64_t)(n / 2), last - col.a + 1));
        const int nb = (int)max((int64_t)0, min((int64_t)(n / 2), last - col.b + 1));
        hit |= tie & (((1u << na) - 1u) | ((1u << nb) - 1u) << (n / 2));
      }
      if (hit) {
        int q = atomicAdd(&ncand, __popc(hit));
        const uint32_t ca = ~(uint32_t)col.a, cb = ~(uint32_t)col.b;
#pragma unroll
        for (int j = 0; j < n; ++j) {
          if (hit >> j & 1) {
            if (q < kCand) cand[q] = (uint64_t)order_of(x[j]) << 32 | (j < n / 2 ? ca - j : cb - (j - n / 2));
            ++q;
          }
        }
      }
    };
    {   // the entries that reach the bound's value
      const uint32_t vo = (uint32_t)(floor_key >> 32);
      const float low = __uint_as_float(__float_as_uint(order_inv(vo == 0x7fffffffu ? 0x80000000u : vo)) & 0xffff0000u);
      const int ne = (it + (1 << ng) - 1) >> ng;   // entries this thread wrote
      uint32_t in = 0;
#pragma unroll
      for (int e = 0; e < kNote / 2; ++e) {
        if (2 * e < ne) {
          const uint32_t v = note[e][tid];
          if (__uint_as_float(v << 16) >= low) in |= 1u << (2 * e);
          if (__uint_as_float(v & 0xffff0000u) >= low) in |= 2u << (2 * e);
        }
      }
      if (ne < 32) in &= (1u << ne) - 1u;
      if (in) {
        int q = atomicAdd(&nsel, __popc(in));
        for (; in; in &= in - 1, ++q)
          if (q < kSel) sel[q] = (__ffs(in) - 1) * NT + tid;
      }
    }
    __syncthreads();
    const int ns = nsel;
    auto collect = [&](uint64_t least) {
      if (ns <= kSel) {
        for (int i = tid; i < ns << ng; i += NT) {
          const int e = sel[i >> ng];
          const int32_t p = p0 + e % NT + ((e / NT << ng) + (i & ((1 << ng) - 1))) * NT;
          if (p < p1) {
            uint32_t words[8];
            load_pair(r, p, words);
            offer(p, words, least);
          }
        }
      } else {   // very many pairs reach the value (a nearly constant row): every thread looks through its own
        for (int32_t p = p0 + tid; p < p1; p += NT) {
          uint32_t words[8];
          load_pair(r, p, words);
          offer(p, words, least);
        }
      }
      __syncthreads();
    };
    collect(floor_key);
    nc = ncand;
    if (nc > kCand) {
      // A few threads own very many large elements.  Bisect on the elements themselves until between k and
      // kCand of them are left; element keys are distinct, so this ends (after at most 64 sweeps).
      uint64_t L = floor_key, H = ~0ull;   // more than kCand elements >= L, fewer than k >= H
      do {
        const uint64_t mid = L + (H - L) / 2;
        __syncthreads();
        if (tid == 0) ncand = 0;
        __syncthreads();
        collect(mid);
        nc = ncand;
        if (nc > kCand) L = mid;
        else if (nc < k) H = mid;
      } while ((nc > kCand || nc < k) && H - L > 1);
    }
    if (nc > kCount) nc = narrow<NT>(cand, nc, cand, k, hist, sh_lo, sh_hi, ncand);
    if (tid < 2) cand[nc + tid] = 0;
    __syncthreads();
  }

  const bool lead = part == 0;
  if (S > 1) {
    // ---- the CTA's list goes to the first CTA of the cluster, which joins the lists
    if (k > 0) {
      uint64_t *dst = cluster.map_shared_rank(lists, 0) + part * k;
      for (int i = tid; i < nc; i += NT) {
        const uint64_t mine = cand[i];
        const int rk = count_larger(cand, nc, mine);
        if (rk < k) dst[rk] = mine;
      }
      for (int i = nc + tid; i < k; i += NT) dst[i] = 0;
    }
    cluster.barrier_arrive();   // (2) everything this CTA had to write is written
    if (!lead) return;
    cluster.barrier_wait();     // (2)
  } else {
    __syncthreads();
  }

  // ---- the row's results
  Soft tot = all_soft[0];
  int32_t cn = all_cnt[0];
  if (S > 1) {   // lane q: CTA q's part
    const bool in = lane < S;
    tot.m = in ? all_soft[lane].m : kLowest;
    tot.s = in ? all_soft[lane].s : 0.f;
    tot.u = in ? all_soft[lane].u : 0.f;
    tot = soft_warp(tot, c);
    cn = __reduce_add_sync(0xffffffffu, in ? all_cnt[lane] : 0);
  }
  const bool bad = !(tot.s <= 3.0e38f);   // NaN or plus infinity in the row
  const bool empty = tot.s == 0.f;        // no finite element
  const float nan = __int_as_float(0x7fffffff);
  const float log_s = bad ? nan : empty ? -INFINITY : logf(tot.s);   // s >= 1
  const float row_max = bad ? nan : empty ? -INFINITY : tot.m;
  if (tid == 0) {
    if (a.row_max) a.row_max[t] = row_max;
    if (a.log_sum) a.log_sum[t] = log_s;
    // u is below zero but for its rounding
    if (a.entropy) a.entropy[t] = bad ? nan : empty ? 0.f : log_s - kLn2 * (fminf(tot.u, 0.f) / tot.s);
    if (a.logprob) {
      float lp = 0.f;   // ignored target
      if (y >= a.V || (bad && y >= 0)) lp = nan;
      else if (y >= 0) lp = xt > -INFINITY ? scaled_diff(xt, row_max, a.scale) - log_s : -INFINITY;
      a.logprob[t] = lp;
    }
    if (RANK && a.rank) a.rank[t] = count && !bad ? cn : -1;
  }
  if (k > 0) {
    auto put = [&](int place, uint64_t e) {
      const bool none = e == 0 || bad;
      const float x = order_inv((uint32_t)(e >> 32));
      a.top_lp[t * k + place] = bad ? nan : none ? -INFINITY : scaled_diff(x, row_max, a.scale) - log_s;
      a.top_id[t * k + place] = none ? -1 : (int32_t)~(uint32_t)e;
    };
    const uint64_t *from = cand;
    int slots = nc, have = nc;
    if (S > 1) {
      // the lists as one; they hold fewer than k elements in all only when the columns run out
      from = lists;
      slots = S * k;
      have = 0;
      for (int base = 0; base < slots; base += NT) have += __syncthreads_count(base + tid < slots && lists[base + tid] != 0);
      if (slots > kCount && have > k) {
        slots = have = narrow<NT>(lists, slots, lists, k, hist, sh_lo, sh_hi, ncand);
        if (tid == 0) lists[slots] = 0;
      } else if (tid == 0 && (slots & 1)) {
        lists[slots] = 0;
      }
      __syncthreads();
    }
    for (int i = tid; i < slots; i += NT) {
      const uint64_t mine = from[i];
      if (mine == 0) continue;
      const int rk = count_larger(from, slots, mine);
      if (rk < k) put(rk, mine);
    }
    for (int i = have + tid; i < k; i += NT) put(i, 0);
  }
}

template <typename T, int NT, bool RANK>
cudaError_t launch_lp(const LpArgs &a, int64_t rows, int S, cudaStream_t st) {
  auto kern = token_logprobs_kernel<T, NT, RANK>;
  if (S > 8) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * S));
  cfg.blockDim = dim3(NT);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)S;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = S > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

// CTAs per row and their size.  Few rows: 256 threads and as many CTAs per row as fill three to an SM (64 rows of
// 1,000,000 bf16, rank and 50 best: 47 us with 6 CTAs, 60 with 8, with 16 of 128 threads 59), as long as a CTA keeps 32 KB
// of the row, since joining the lists costs 2 to 3 us (200 rows of 5,000 fp32: 8.2 us with one CTA, 9.8 with two; one row
// of 100,000 bf16: 11.4 with 6, 11.5 with 16).  Many rows: one CTA of 128 threads each, of which seven share an SM, so that
// the end of one row, which is latency, hides behind the passes of six others (4096 rows of 20,000 fp32: 76 us, with
// 256 threads 108 us).
template <typename T>
cudaError_t dispatch_lp(const LpArgs &a, int64_t rows, cudaStream_t st) {
  const int64_t bytes = (int64_t)a.V * (int64_t)sizeof(T);
  if (rows > 3 * kSMs) return a.rank ? launch_lp<T, 128, true>(a, rows, 1, st) : launch_lp<T, 128, false>(a, rows, 1, st);
  int S = 1;
  while (S < kRowClusterMax && rows * (S + 1) <= 3 * kSMs && bytes / (S + 1) >= 32768) ++S;
  while (S > 1 && S * a.k > kLists) --S;   // the first CTA holds the lists of all
  return a.rank ? launch_lp<T, 256, true>(a, rows, S, st) : launch_lp<T, 256, false>(a, rows, S, st);
}

// ---- backward ---------------------------------------------------------------------------------------------------------
struct LpGradArgs {
  const void *x;
  int64_t stride;
  const void *y;
  int32_t y64, V;
  float scale;
  const float *row_max, *log_sum, *entropy, *g, *h;
  void *dx;
  int64_t dstride;
  int64_t rows;
  int32_t chunks;   // CTAs per row
};

// One CTA takes every `chunks`-th run of NT pairs of a row.  log p is computed from the row's maximum and log
// sum as the forward pass stored them, so it has the forward pass's accuracy whatever the size of the scores:
//   t = c (x - max) - log2 sum = log2 p,   d = p (A t + K),   A = -h scale log 2,  K = -(g + h H) scale.
// An excluded column has t = -inf: 2^t is zero and the clamp keeps the product zero.
// Memory bound: 2048 x 100,000 bf16 in 136 us, 6.0 TB/s of reads and writes (92 % of the copy rate); with 13 CTAs a row
// instead of 3, each thread had two pairs to spread its set-up over, and it took 148 us.
template <typename T, typename TO, int NT>
__global__ void __launch_bounds__(NT) token_logprobs_grad_kernel(const LpGradArgs a) {
  constexpr int n = 2 * El<T>::kPer16, kAhead = 2;
  const int64_t t = blockIdx.x;
  const int ch = (int)blockIdx.y;
  const RowChunks<T> r(static_cast<const T *>(a.x) + t * a.stride, a.V);
  TO *drow = static_cast<TO *>(a.dx) + t * a.dstride;
  const int32_t step = a.chunks * NT;
  PairMap<T, TO, kAhead> map(r, drow, ch * NT + (int32_t)threadIdx.x, step);
  map.start(r.pairs);
  float mx = a.row_max[t], ls = a.log_sum[t];
  const int64_t y = a.y ? load_id(a.y, t, a.y64) : -1;
  const bool has_y = y >= 0 && y < a.V;
  const float xy = has_y ? El<T>::load(r.row + y) : 0.f;   // before anything is written: the gradient may lie in its place
  const float g = a.g && has_y ? a.g[t] : 0.f;
  const float h = a.h ? a.h[t] : 0.f, H = a.h ? a.entropy[t] : 0.f;
  const bool empty = ls == -INFINITY;
  if (empty) mx = 0.f, ls = INFINITY;   // no column left: p = 0 everywhere
  const float c = a.scale * kLog2e;
  const f32x2 c2 = mk2(c, c), nmx = mk2(-mx, -mx), nls = mk2(-ls * kLog2e, -ls * kLog2e);
  const float A = -h * a.scale * kLn2, K = -fmaf(h, H, g) * a.scale;
  const f32x2 A2 = mk2(A, A), K2 = mk2(K, K);
  const int32_t ygroup = has_y && !empty ? (int32_t)((y + r.lead) / (32 * n)) : -1;
  map.run(
      r.pairs,
      [&](int32_t, float(&x)[n]) {
#pragma unroll
        for (int j = 0; j < n; j += 2) {
          float t0, t1;
          un2(fma2(add2(mk2(x[j], x[j + 1]), nmx), c2, nls), t0, t1);
          t0 = max_nan(t0, kFloor2);
          t1 = max_nan(t1, kFloor2);
          un2(mul2(mk2(ex2(t0), ex2(t1)), fma2(mk2(t0, t1), A2, K2)), x[j], x[j + 1]);
        }
      },
      [&](int32_t q) {
        if (q >> 5 == ygroup && y >= r.first(r.chunk(q)) &&
            (y < r.first(r.chunk(q) + 1) || (y >= r.first(r.chunk(q) + 32) && y < r.first(r.chunk(q) + 33)))) {
          // the thread that wrote the target's column writes it again, with the target's own term
          const float t0 = max_nan(fmaf(xy - mx, c, -ls * kLog2e), kFloor2);
          drow[y] = El<TO>::from(fmaf(ex2(t0), fmaf(t0, A, K), g * a.scale));
        }
      });
}

template <typename T, typename TO>
cudaError_t launch_lp_grad(LpGradArgs a, cudaStream_t st) {
  constexpr int NT = 256;
  // CTAs per row: 32 per SM in all (2048 rows of 100,000 bf16 136 us, with 128 per SM 140), as long as a thread keeps two
  // pairs (one row of 100,000 bf16: 3.4 us, with four 4.5)
  const int64_t pairs = ((int64_t)a.V + El<T>::kPer16) / (2 * El<T>::kPer16) + 1, most = (pairs + 2 * NT - 1) / (2 * NT);
  int64_t chunks = (32 * kSMs + a.rows - 1) / a.rows;
  if (chunks > most) chunks = most;
  if (chunks > 65535) chunks = 65535;
  a.chunks = (int32_t)chunks;
  token_logprobs_grad_kernel<T, TO, NT><<<dim3((unsigned)a.rows, (unsigned)chunks), NT, 0, st>>>(a);
  return cudaGetLastError();
}

bool aligned_to(const void *p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; }

}  // namespace
}  // namespace tsid

using namespace tsid;

extern "C" {

tsid_status_t tsid_token_logprobs(int64_t n_rows, int32_t n_cols, const void *d_logits, int32_t logits_dtype,
                                  int64_t row_stride, float scale, const void *d_targets_or_null, int32_t targets_i64,
                                  int32_t top_k, float *d_logprob_or_null, float *d_entropy_or_null,
                                  float *d_row_max_or_null, float *d_log_sum_or_null, int32_t *d_rank_or_null,
                                  float *d_top_logprob, int32_t *d_top_id, void *stream) {
  if (n_rows < 0 || n_cols < 1) return refuse(TSID_ERR_INVALID_ARG, "n_rows must be >= 0 and n_cols >= 1");
  if (!dtype_ok(logits_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad logits dtype");
  if (!(scale >= kScaleMin) || !(scale <= kScaleMax)) return refuse(TSID_ERR_INVALID_ARG, "scale must be in [1e-20, 1e20]");
  if (top_k < 0 || top_k > TSID_TOP_MAX || top_k > n_cols)
    return refuse(TSID_ERR_INVALID_ARG, "top_k must be in [0, min(TSID_TOP_MAX, n_cols)]");
  if (n_rows == 0) return TSID_OK;
  if (n_rows > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
  if (!d_logits || !aligned_to(d_logits, dtype_bytes(logits_dtype)) || (n_rows > 1 && row_stride < n_cols))
    return refuse(TSID_ERR_INVALID_ARG, "logits: null, misaligned, or row_stride smaller than n_cols");
  if (top_k > 0 && (!d_top_logprob || !d_top_id)) return refuse(TSID_ERR_INVALID_ARG, "top_k > 0 needs both top arrays");
  if ((d_logprob_or_null || d_rank_or_null) && !d_targets_or_null)
    return refuse(TSID_ERR_INVALID_ARG, "log probabilities and ranks need targets");
  LpArgs a = {d_logits, row_stride, d_targets_or_null, targets_i64, n_cols, top_k, scale, d_logprob_or_null,
              d_entropy_or_null, d_row_max_or_null, d_log_sum_or_null, d_rank_or_null, d_top_logprob, d_top_id};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = logits_dtype == TSID_DT_F32    ? dispatch_lp<float>(a, n_rows, st)
                  : logits_dtype == TSID_DT_BF16 ? dispatch_lp<__nv_bfloat16>(a, n_rows, st)
                                                 : dispatch_lp<__half>(a, n_rows, st);
  return e == cudaSuccess ? TSID_OK : refuse(TSID_ERR_CUDA, cudaGetErrorString(e));
}

tsid_status_t tsid_token_logprobs_grad(int64_t n_rows, int32_t n_cols, const void *d_logits, int32_t logits_dtype,
                                       int64_t row_stride, float scale, const void *d_targets_or_null,
                                       int32_t targets_i64, const float *d_row_max, const float *d_log_sum,
                                       const float *d_entropy_or_null, const float *d_g_logprob_or_null,
                                       const float *d_g_entropy_or_null, void *d_grad, int32_t grad_dtype,
                                       int64_t grad_stride, void *stream) {
  if (n_rows < 0 || n_cols < 1) return refuse(TSID_ERR_INVALID_ARG, "n_rows must be >= 0 and n_cols >= 1");
  if (!dtype_ok(logits_dtype) || !dtype_ok(grad_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad dtype");
  if (grad_dtype != logits_dtype && grad_dtype != TSID_DT_F32)
    return refuse(TSID_ERR_UNSUPPORTED, "the gradient has the logits' dtype or fp32");
  if (!(scale >= kScaleMin) || !(scale <= kScaleMax)) return refuse(TSID_ERR_INVALID_ARG, "scale must be in [1e-20, 1e20]");
  if (n_rows == 0) return TSID_OK;
  if (n_rows > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
  if (!d_logits || !aligned_to(d_logits, dtype_bytes(logits_dtype)) || (n_rows > 1 && row_stride < n_cols))
    return refuse(TSID_ERR_INVALID_ARG, "logits: null, misaligned, or row_stride smaller than n_cols");
  if (!d_grad || !aligned_to(d_grad, dtype_bytes(grad_dtype)) || (n_rows > 1 && grad_stride < n_cols))
    return refuse(TSID_ERR_INVALID_ARG, "grad: null, misaligned, or grad_stride smaller than n_cols");
  if (!d_row_max || !d_log_sum) return refuse(TSID_ERR_INVALID_ARG, "row_max and log_sum are needed");
  if (d_g_logprob_or_null && !d_targets_or_null) return refuse(TSID_ERR_INVALID_ARG, "a log probability gradient needs targets");
  if (d_g_entropy_or_null && !d_entropy_or_null) return refuse(TSID_ERR_INVALID_ARG, "an entropy gradient needs the entropies");
  if (d_grad == d_logits && (grad_dtype != logits_dtype || grad_stride != row_stride))
    return refuse(TSID_ERR_INVALID_ARG, "in place needs the same dtype and stride");
  LpGradArgs a = {d_logits, row_stride, d_targets_or_null, targets_i64, n_cols, scale, d_row_max, d_log_sum,
                  d_entropy_or_null, d_g_logprob_or_null, d_g_entropy_or_null, d_grad, grad_stride, n_rows, 1};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (logits_dtype == TSID_DT_F32) e = launch_lp_grad<float, float>(a, st);
  else if (logits_dtype == TSID_DT_BF16)
    e = grad_dtype == TSID_DT_F32 ? launch_lp_grad<__nv_bfloat16, float>(a, st) : launch_lp_grad<__nv_bfloat16, __nv_bfloat16>(a, st);
  else
    e = grad_dtype == TSID_DT_F32 ? launch_lp_grad<__half, float>(a, st) : launch_lp_grad<__half, __half>(a, st);
  return e == cudaSuccess ? TSID_OK : refuse(TSID_ERR_CUDA, cudaGetErrorString(e));
}

}  // extern "C"
