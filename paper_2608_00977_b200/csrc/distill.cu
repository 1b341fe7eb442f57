// Distillation from a teacher's top columns: loss and gradient in one launch.
//
// A row has student scores x_v, z = scale x, q = softmax(z), and a teacher's list of K distinct columns with
// log probabilities l_k (a negative id is an empty place).
//   RENORM: p_k = softmax of l over the list,  L = sum_k p_k (log p_k - log q_k)
//   TAIL:   p_k = e^{l_k}; everything outside the list is one more outcome with p_T = max(0, 1 - sum p_k) and
//           q_T = sum of q outside the list:  L = sum_k p_k (l_k - log q_k) + p_T (log p_T - log q_T)
//   dL/dz_v = W q_v - p_v [v in list] - [v not in list] p_T q_v / q_T,  W = sum of the p that take part.
//
// One CTA or cluster of CTAs per row: a first pass over the row for the softmax sums, a join over the cluster through
// distributed shared memory, the loss, and a second pass that writes the gradient.  The launch keeps the rows that
// are being worked on well inside L2, so the second pass reads them from there and the row crosses the memory bus
// once.  The sum outside the list is formed by leaving the list's columns out, not by subtracting them, so a small
// tail keeps its accuracy; a warp finds the few chunks that hold a listed column with one bit per 16-byte chunk, by its
// number modulo 32 kMarkWords, in shared memory.
//
// What bounds it (times of the kernel alone; a call in a sequence of calls takes 2 to 12 us more): 2048 x 100,000 bf16 with 64
// listed columns takes 197 us against 125 us for one read and one write at the copy rate (6.55 TB/s), the loss alone 103 us.
// DRAM traffic is that minimum (428 MB read, the gradient written).  No unit is full: issue slots 58 %, the 2^x unit 50 %
// (two 2^x and some 18 instructions per element), memory 64 %, 44 % of the warps active; a CTA's two passes follow each other
// with a join between them, in which it loads nothing.  The time is linear in the rows (1960 to 2400 rows: 0.096 us each, no
// step at a whole wave).  How far the student is makes 1 %.  Tried and slower: the row held in shared memory
// between the passes by clusters of 4 to 8 CTAs (258 - 310 us: short CTAs, whose set-up and cluster barriers outweigh the
// saved L2 reads), one CTA of 512 threads a row (201 us).
#include <cooperative_groups.h>

#include <algorithm>

#include "rows.cuh"

namespace cg = cooperative_groups;

namespace tsid {
namespace {

#define CK(x)                         \
  do {                                \
    cudaError_t e_ = (x);             \
    if (e_ != cudaSuccess) return e_; \
  } while (0)

constexpr int kListMax = TSID_TOP_MAX;
constexpr int kMarkWords = 256;   // words of 32 chunks each

struct DistillArgs {
  const void *x;
  int64_t stride;
  const int32_t *ids;
  const float *tlp;
  const float *weight;
  float *loss;
  void *dx;
  int64_t dstride;
  float scale;
  int32_t V, k, tail;
};

struct Sum {
  float m, s;   // sum of 2^(c (x - m))
};
__device__ __forceinline__ Sum sum_warp(const Sum &v, float c) {
  Sum r;
  r.m = warp_max(v.m);
  r.s = v.s * ex2(fmaxf((v.m - r.m) * c, kFloor2));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
  return r;
}
__device__ __forceinline__ float add_warp(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What a CTA contributes to its row: the columns of its part of the row outside the list, and those in it.
struct Part {
  Sum rest, listed;
  float W;      // sum of p
  float pl;     // sum of p l
  float px;     // sum of p (x - listed.m) / 2 (halves: see half_diff)
  float bad;    // an id beyond the columns (every CTA sees all ids)
};

template <typename T, typename TO, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) distill_kernel(const DistillArgs a) {
  constexpr int n = 2 * El<T>::kPer16;   // elements of a pair
  constexpr int h = n / 2;
  constexpr int NW = NT / 32;
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int64_t t = (int64_t)blockIdx.x / S;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;

  // the listed columns in this CTA's part (id -1: empty place, or elsewhere): log probability, probability, score and
  // gradient
  __shared__ int32_t id_s[kListMax], next_s[kListMax];
  __shared__ float l_s[kListMax], p_s[kListMax], x_s[kListMax], v_s[kListMax];
  __shared__ __align__(8) uint32_t mark[kMarkWords];
  __shared__ int32_t head[kMarkWords];
  __shared__ Sum sh_sum[NW];
  __shared__ Part mine;
  __shared__ struct { float mx, total, W, pT, rest_m, rest_s, rest_f; } row;   // rest_s about rest_m, rest_f = 2^(c (rest_m - mx))
  __shared__ int32_t beyond;
  extern __shared__ __align__(16) unsigned char dyn[];   // the ring
  static_assert(kListMax <= NT, "a thread takes one place of the list");

  const RowChunks<T> r(static_cast<const T *>(a.x) + t * a.stride, a.V);
  const int32_t per = ((r.pairs >> 5) + S - 1) / S * 32;   // pairs of a CTA: whole groups of 32
  const int32_t p0 = min(part * per, r.pairs), p1 = min(p0 + per, r.pairs);
  const float c = a.scale * kLog2e;
  const int k = a.k;
  PairStream<T, NT> stream(r, *reinterpret_cast<PairRing<NT> *>(dyn), p0 + tid, p1);
  const float wt = (a.weight ? a.weight[t] : 1.f) * a.scale;

  // ---- the list: columns are chained by the word of marks their chunk belongs to
  int32_t my_id = -1;
  float my_l = -INFINITY;
  if (tid < k) {   // kListMax <= NT
    my_id = a.ids[t * k + tid];
    my_l = a.tlp[t * k + tid];
  }
  for (int i = tid; i < kMarkWords; i += NT) {
    mark[i] = 0;
    head[i] = -1;
  }
  if (tid == 0) beyond = 0;
  __syncthreads();
  const int64_t lo = r.first(2 * p0), hi = r.first(2 * p1);   // the columns of this CTA's part
  const bool own = my_id >= lo && my_id < hi && my_id >= 0 && my_id < a.V;
  const int32_t my_chunk = own ? (int32_t)(((int64_t)my_id + r.lead) / h) : 0;
  const uint32_t my_word = (uint32_t)(my_chunk >> 5) & (kMarkWords - 1);
  float my_x = -INFINITY;
  if (own) my_x = El<T>::load(r.row + my_id);
  if (tid < k) {
    if (my_id >= a.V) beyond = 1;
    id_s[tid] = own ? my_id : -1;
    l_s[tid] = my_id >= 0 && my_id < a.V ? my_l : -INFINITY;
    if (own) next_s[tid] = atomicExch(&head[my_word], tid);
  }
  __syncthreads();
  bool again = false;   // of a repeated id the first place counts
  if (own) {
    for (int i = head[my_word]; i >= 0; i = next_s[i]) again |= i < tid && id_s[i] == my_id;
    if (!again) atomicOr(&mark[my_word], 1u << (my_chunk & 31));
  }
  float shift = 0.f;
  if (!a.tail) {   // the list's own normalisation (over all of it: a repeated id is looked for in the whole list)
    __shared__ float sh_list[2];
    __shared__ int32_t all_s[kListMax];
    if (tid < k) all_s[tid] = my_id;
    __syncthreads();
    if (tid < k && my_id >= 0 && my_id < a.V && !own)   // other CTAs' columns: the same first-place rule
      for (int i = 0; i < tid; ++i) again |= all_s[i] == my_id;
    if (tid < k && again) l_s[tid] = -INFINITY;
    __syncthreads();
    if (w == 0) {
      float lm = -INFINITY;
      for (int i = lane; i < k; i += 32) lm = max_nan(lm, l_s[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) lm = max_nan(lm, __shfl_xor_sync(0xffffffffu, lm, o));
      float ls = 0.f;
      if (lm != -INFINITY)
        for (int i = lane; i < k; i += 32) ls += expf(l_s[i] - lm);
      ls = add_warp(ls);
      if (lane == 0) sh_list[0] = lm == -INFINITY ? 0.f : lm + logf(ls);
    }
    __syncthreads();
    shift = sh_list[0];
  }
  const bool counts = own && !again;
  if (own && again) id_s[tid] = -1;
  __syncthreads();

  // ---- first pass: the sum over the columns outside the list
  const f32x2 c2 = mk2(c, c);
  RunningSoft<n, false> sums(a.scale);
  float top = -INFINITY;   // its largest
  // calls f(i, j, u) for the listed columns of pair p: place i of the list, element u of the pair's chunk j
  auto listed_of = [&](int32_t p, auto f) {
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      const int32_t ch = r.chunk(p) + 32 * j;
      const uint32_t word = (uint32_t)(ch >> 5) & (kMarkWords - 1);
      if (!(mark[word] >> lane & 1u)) continue;
      const int32_t e0 = (int32_t)r.first(ch);
      for (int i = head[word]; i >= 0; i = next_s[i]) {
        const uint32_t u = (uint32_t)(id_s[i] - e0);
        if (id_s[i] >= 0 && u < (uint32_t)h) f(i, j, u);
      }
    }
  };
  auto marked = [&](int32_t p) {   // the pair's chunks are bit `lane` of two neighbouring words
    const uint2 g = *reinterpret_cast<const uint2 *>(&mark[2 * (p >> 5) & (kMarkWords - 1)]);
    return ((g.x | g.y) >> lane) & 1u;
  };
  auto take = [&](int32_t p, const uint32_t(&raw)[8]) {
    float x[n];
    unpack<T, 8>(raw, x);
    const float cm = fmaxf(chunk_max<T>(raw[0], raw[1], raw[2], raw[3]), chunk_max<T>(raw[4], raw[5], raw[6], raw[7]));
    top = fmaxf(top, cm);
    sums.take(x, cm);
  };
  // the listed columns are struck out of the staged pair before it is read
  stream.run(take, [&](int32_t p, uint32_t slot) {
    if (marked(p))
      listed_of(p, [&](int, int j, uint32_t u) {
        const uint32_t at = slot + (uint32_t)(j * NT * 16) + u * (uint32_t)sizeof(T);
        if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(El<T>::kFill) : "memory");
        else asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((uint16_t)(El<T>::kFill & 0xffffu)) : "memory");
      });
  });
  // ---- this CTA's listed columns (their scores were fetched before the pass)
  const float my_ln = my_l - shift, my_p = counts ? expf(my_ln) : 0.f;
  if (tid < k) {
    l_s[tid] = counts ? my_ln : 0.f;
    p_s[tid] = my_p;
    x_s[tid] = counts ? my_x : -INFINITY;
  }
  {
    const Soft part_sum = sums.result(top);
    Sum v = {part_sum.m, part_sum.s};
    v = sum_warp(v, c);
    if (lane == 0) sh_sum[w] = v;
  }
  __syncthreads();
  if (w == NW - 1) {   // meanwhile, the listed columns
    Part q;
    q.listed.m = kLowest;
    for (int i = lane; i < k; i += 32) q.listed.m = fmaxf(q.listed.m, x_s[i]);
    q.listed.m = warp_max(q.listed.m);
    q.listed.s = q.W = q.pl = q.px = 0.f;
    for (int i = lane; i < k; i += 32) {
      const float p = p_s[i], d = half_diff(x_s[i], q.listed.m);
      q.listed.s += ex2(max_nan(2.f * d * c, kFloor2));
      q.W += p;
      if (p > 0.f || p != p) {
        q.pl += p * l_s[i];
        q.px += p * d;
      }
    }
    q.listed.s = add_warp(q.listed.s);
    q.W = add_warp(q.W);
    q.pl = add_warp(q.pl);
    q.px = add_warp(q.px);
    if (lane == 0) {
      mine.listed = q.listed;
      mine.W = q.W;
      mine.pl = q.pl;
      mine.px = q.px;
      mine.bad = beyond ? 1.f : 0.f;
    }
  }
  if (w == 0) {
    Sum q;
    q.m = kLowest;
    q.s = 0.f;
    if (lane < NW) q = sh_sum[lane];
    q = sum_warp(q, c);
    if (lane == 0) mine.rest = q;
  }
  __syncthreads();

  // the second pass's first pairs are on their way while the row is joined
  TO *const drow = static_cast<TO *>(a.dx) + t * a.dstride;
  PairMap<T, TO, 2> map(r, drow, p0 + tid, NT);
  if (a.dx) map.start(p1);

  // ---- join over the cluster, in the order of its CTAs, about the common maximum: by one warp of each CTA
  if (S > 1) cluster.sync();
  if (w == 0) {
    Part o;   // lane q: CTA q's part
    o.rest.m = o.listed.m = kLowest;
    o.rest.s = o.listed.s = o.W = o.pl = o.px = o.bad = 0.f;
    if (lane < S) o = S > 1 ? *cluster.map_shared_rank(&mine, lane) : mine;
    const Sum rest = sum_warp(o.rest, c), listed = sum_warp(o.listed, c);
    const float W = add_warp(o.W);
    const float mx = fmaxf(rest.m, listed.m);
    const float rest_f = ex2(fmaxf((rest.m - mx) * c, kFloor2)), rest_s = rest.s * rest_f;
    const float total = rest_s + listed.s * ex2(fmaxf((listed.m - mx) * c, kFloor2));
    const float pT = a.tail && rest.s > 0.f ? fmaxf(1.f - W, 0.f) : 0.f;   // no column outside the list: no such outcome
    if (lane == 0) row = {mx, total, W, pT, rest.m, rest.s, rest_f};
    if (part == 0 && a.loss) {
      const float pl = add_warp(o.pl), bad = add_warp(o.bad);
      const float px = add_warp(o.W == 0.f ? o.px : fmaf(o.W, half_diff(o.listed.m, listed.m), o.px));
      if (lane == 0) {
        // sum p (l - scale (x - mx) + log total)
        float L = W > 0.f || W != W ? pl - 2.f * a.scale * fmaf(W, half_diff(listed.m, mx), px) + W * logf(total) : 0.f;
        // one logarithm of the ratio keeps a small loss accurate; a tail below fp32's range leaves its reference out of it
        const bool tiny = rest_s <= 1e-30f;
        if (pT > 0.f) L += pT * (logf(pT * (total / (tiny ? rest.s : rest_s))) - (tiny ? scaled_diff(rest.m, mx, a.scale) : 0.f));
        a.loss[t] = bad != 0.f ? __int_as_float(0x7fffffff) : total == 0.f ? 0.f : L + 0.f * total;
      }
    }
  }
  __syncthreads();
  if (S > 1) cluster.barrier_arrive();   // this CTA has read what it needs of the others
  const float mx = row.mx, total = row.total, pT = row.pT, Wall = row.W + row.pT;
  const bool empty = total == 0.f;

  // ---- second pass: the gradient
  if (a.dx) {
    // factors of 2^(c (x - mx)) of a listed column, and of 2^(c (x - rest_m)) of any other, whose share of the tail
    // matters even where the whole tail is nothing beside the row; a row without any column left gets zeros
    const float in_list = empty ? 0.f : Wall / total * wt;
    const float outside = empty ? 0.f : (Wall * row.rest_f / total - (pT > 0.f ? pT / row.rest_s : 0.f)) * wt;
    const f32x2 nrm = mk2(-row.rest_m, -row.rest_m), outside2 = mk2(outside, outside);
    // A 16-bit gradient has room for a shorter form: the factor goes into the exponent, outside 2^(c (x - rest_m)) =
    // 2^(c x + fold), one multiply-add and one 2^x per element.  The exponent's rounding is at most 2^-16 of the result
    // while |fold| is at most 256, against the 2^-9 (bf16) or 2^-11 (fp16) of the store.
    const float fold = log2f(outside) - row.rest_m * c;
    const bool folded = sizeof(TO) == 2 && outside > 0.f && fabsf(fold) <= 256.f;
    const f32x2 fold2 = mk2(fold, fold);
    if (counts) v_s[tid] = ex2(max_nan((my_x - mx) * c, kFloor2)) * in_list - (empty ? 0.f : my_p * wt);
    __syncthreads();
    map.run(
        p1,
        [&](int32_t, float(&x)[n]) {
          if (folded) {
#pragma unroll
            for (int j = 0; j < n; j += 2) {
              float t0, t1;
              un2(fma2(mk2(x[j], x[j + 1]), c2, fold2), t0, t1);
              x[j] = ex2(t0);
              x[j + 1] = ex2(t1);
            }
          } else {
#pragma unroll
            for (int j = 0; j < n; j += 2) {
              float t0, t1;
              un2(mul2(add2(mk2(x[j], x[j + 1]), nrm), c2), t0, t1);
              un2(mul2(mk2(ex2(t0), ex2(t1)), outside2), x[j], x[j + 1]);
            }
          }
        },
        [&](int32_t p) {   // the thread that wrote a listed column writes it again
          if (marked(p))
            listed_of(p, [&](int i, int, uint32_t) { drow[id_s[i]] = El<TO>::from(v_s[i]); });
        });
  }
  if (S > 1) cluster.barrier_wait();   // no CTA leaves while its part may still be read
}

template <typename T, typename TO, int NT>
cudaError_t launch_distill(const DistillArgs &a, int64_t rows, int S, cudaStream_t st) {
  auto kern = distill_kernel<T, TO, NT>;
  if (S > 8) CK(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  static_assert(sizeof(PairRing<NT>) <= 48 * 1024, "above that a kernel has to opt in");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * S));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = sizeof(PairRing<NT>);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)S;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = S > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

// CTAs per row and their size (1024 threads an SM).
//   Few rows: a row is spread over CTAs of 128 threads as long as a CTA keeps 4 KB of it and they cover the SMs less than
// wholly, 7 of 8 places (130 rows of 20,001 fp32: 13.2 us with 7 CTAs a row, 23.3 with one; 300 rows of 20,000 bf16: 16.0
// with 3, 21.4 with one, and 23.0 with 4, which need a second wave).  Clusters of more than 8 leave more places unused
// and get 6 of 8 (74 rows of 100,000 bf16: 15.7 us with 12 CTAs, 23.0 with 14).
//   Rows being worked on beyond kL2Rows bytes would be read from memory twice, so they are spread until they fit (2048
// rows of 100,000 bf16: 196 us with 3 CTAs, 79 MB, against 218 with 2 and 233 with one; 2048 rows of 60,000, 71 MB with 2:
// 127 us, with 3 135).
//   Where that gives the largest cluster, CTAs of 256 threads (one row of 100,000: 9.2 us, with 128 threads 9.7; 300 rows
// of 1,000,000: 283 and 316 us).  Elsewhere the smaller ones end more evenly (4096 rows of 8,500 bf16: 94 us, with 256
// threads 132).
constexpr int64_t kL2Rows = 80 << 20;
template <typename T, typename TO>
cudaError_t dispatch_distill(const DistillArgs &a, int64_t rows, cudaStream_t st) {
  const int64_t bytes = (int64_t)a.V * (int64_t)sizeof(T);
  auto ctas_of = [&](int NT) {
    const int64_t resident = kSMs * (1024 / NT);
    int64_t S = 1;
    while (S < kRowClusterMax) {
      const bool fits = rows * (S + 1) <= (S < 8 ? 7 : 6) * resident / 8, wide = bytes / (S + 1) >= 32 * NT;
      if (!(fits && wide) && std::min(rows, resident / S) * bytes <= kL2Rows) break;
      ++S;
    }
    return (int)S;
  };
  const int S = ctas_of(128);
  return S < kRowClusterMax ? launch_distill<T, TO, 128>(a, rows, S, st) : launch_distill<T, TO, 256>(a, rows, ctas_of(256), st);
}

bool aligned_to(const void *p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; }

}  // namespace
}  // namespace tsid

using namespace tsid;

extern "C" {

tsid_status_t tsid_distill(int64_t n_rows, int32_t n_cols, const void *d_logits, int32_t logits_dtype,
                           int64_t row_stride, float scale, int32_t top_k, const int32_t *d_teacher_id,
                           const float *d_teacher_logprob, int32_t mode, const float *d_weight_or_null,
                           float *d_loss_or_null, void *d_grad_or_null, int32_t grad_dtype, int64_t grad_stride,
                           void *stream) {
  if (n_rows < 0 || n_cols < 1) return refuse(TSID_ERR_INVALID_ARG, "n_rows must be >= 0 and n_cols >= 1");
  if (!dtype_ok(logits_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad logits dtype");
  if (!(scale >= kScaleMin) || !(scale <= kScaleMax)) return refuse(TSID_ERR_INVALID_ARG, "scale must be in [1e-20, 1e20]");
  if (top_k < 1 || top_k > TSID_TOP_MAX) return refuse(TSID_ERR_INVALID_ARG, "top_k must be in [1, TSID_TOP_MAX]");
  if (mode != TSID_DISTILL_RENORM && mode != TSID_DISTILL_TAIL) return refuse(TSID_ERR_INVALID_ARG, "bad mode");
  if (d_grad_or_null) {
    if (!dtype_ok(grad_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad grad dtype");
    if (grad_dtype != logits_dtype && grad_dtype != TSID_DT_F32)
      return refuse(TSID_ERR_UNSUPPORTED, "the gradient has the logits' dtype or fp32");
    if (n_rows > 0 && (!aligned_to(d_grad_or_null, dtype_bytes(grad_dtype)) || (n_rows > 1 && grad_stride < n_cols)))
      return refuse(TSID_ERR_INVALID_ARG, "grad: misaligned, or grad_stride smaller than n_cols");
    if (d_grad_or_null == d_logits && (grad_dtype != logits_dtype || grad_stride != row_stride))
      return refuse(TSID_ERR_INVALID_ARG, "in place needs the same dtype and stride");
  }
  if (n_rows == 0) return TSID_OK;
  if (!d_loss_or_null && !d_grad_or_null) return refuse(TSID_ERR_INVALID_ARG, "neither a loss nor a gradient is asked for");
  if (n_rows > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 rows");
  if (!d_logits || !aligned_to(d_logits, dtype_bytes(logits_dtype)) || (n_rows > 1 && row_stride < n_cols))
    return refuse(TSID_ERR_INVALID_ARG, "logits: null, misaligned, or row_stride smaller than n_cols");
  if (!d_teacher_id || !d_teacher_logprob) return refuse(TSID_ERR_INVALID_ARG, "the teacher's ids and log probabilities are needed");
  DistillArgs a = {d_logits, row_stride, d_teacher_id, d_teacher_logprob, d_weight_or_null, d_loss_or_null,
                   d_grad_or_null, grad_stride, scale, n_cols, top_k, mode == TSID_DISTILL_TAIL ? 1 : 0};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = d_grad_or_null && grad_dtype == TSID_DT_F32;
  cudaError_t e;
  if (logits_dtype == TSID_DT_F32) e = dispatch_distill<float, float>(a, n_rows, st);
  else if (logits_dtype == TSID_DT_BF16)
    e = wide ? dispatch_distill<__nv_bfloat16, float>(a, n_rows, st) : dispatch_distill<__nv_bfloat16, __nv_bfloat16>(a, n_rows, st);
  else
    e = wide ? dispatch_distill<__half, float>(a, n_rows, st) : dispatch_distill<__half, __half>(a, n_rows, st);
  return e == cudaSuccess ? TSID_OK : refuse(TSID_ERR_CUDA, cudaGetErrorString(e));
}

}  // extern "C"
