// Factor rows of a batch of ids, and the gradient of the table by sorted ids.
//
//   out[t, :]   = scale * table[ids[t], :]
//   dtable[v,:] = scale * sum over t with ids[t] = v of dout[t, :]
//
// Both move rows and compute next to nothing, so memory bounds them.  The gradient sorts (id, position) pairs
// by id, stably, after which the rows of one id are a run of the sorted list; runs are
// summed in fp32 in list order: a group of lanes sums `run` consecutive places in registers, the groups of a CTA
// join the runs that cross group borders through shared memory, and runs that cross CTA borders are joined by a
// last kernel from one partial row per CTA.  The order of every addition depends on the ids, the sizes, the types
// and the layout alone (the lanes that share a row, and with them the borders between groups, follow from the widest
// access that the rows' alignment allows): no float atomics, the same call gives the same bits, and a popular id is
// spread over as many groups as it has places.
//
// Measured on one B200 (6.55 TB/s copy rate; times of the kernels alone, a call in a sequence of calls takes 1 to 10 us more).
// Lookup of 1M x 128 bf16: 83 us, 6.2 TB/s (95 %); rows that are no multiple of 8 bytes go element by element and are bound by
// instructions (1M x 125 bf16 255 us, fp32 204).  Gradient: 1M tokens x 128 bf16 into a table of 1M rows fp32 188 us (118 us
// for one read and one write): 50 us of sorting, in which memory idles, 125 us of sums and zeroing at 6.2 TB/s, 10 us of
// joining; accumulating costs the read of the named rows (with ids spread evenly 237 us, overwriting 184).  65,536 x 64 bf16,
// 100,000 rows: 33 us (5.3), nearly all latency of the sort (17 us), the sums (8) and the join (4).  129 x 33 fp32, 2,000
// rows: 6.2 us in one launch.
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

__device__ __forceinline__ int64_t load_id(const void *ids, int64_t t, int is64) {
  return is64 ? static_cast<const int64_t *>(ids)[t] : (int64_t)static_cast<const int32_t *>(ids)[t];
}

// The VE elements of a row that a lane works on.  WIDE: consecutive ones, moved by 16- or 8-byte accesses (the launcher
// checked sizes and alignment).  Otherwise every cs-th element, so that the lanes of a group touch consecutive elements
// of any alignment; those past the row's end are left out.
struct Slice {
  int e, cs, dim;   // first element, distance to the next, row length
};
// Indices are 32-bit and run past the row's end by less than the elements of one step of a group, 32 lanes x 8.
constexpr int32_t kRowMax = 2147483647 - 1023;
template <typename T, int VE, bool WIDE>
struct Elems {
  static constexpr int kWords = WIDE ? VE * (int)sizeof(T) / 4 : VE;
  uint32_t w[kWords];   // as loaded; unpacked when needed
  __device__ __forceinline__ void load(const T *row, const Slice &s) {
    if constexpr (WIDE) {
      const char *p = reinterpret_cast<const char *>(row + s.e);
      if constexpr (kWords % 4 == 0) {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) ld16(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3], p + 16 * i);
      } else {
        static_assert(kWords == 2, "8 bytes");
        asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
      }
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        w[i] = s.e + i * s.cs < s.dim ? __float_as_uint(El<T>::load(row + s.e + i * s.cs)) : 0u;
    }
  }
  __device__ __forceinline__ void get(float (&x)[VE]) const {
    if constexpr (WIDE) {
      unpack<T, kWords>(w, x);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = __uint_as_float(w[i]);
    }
  }
  static __device__ __forceinline__ void store(T *row, const Slice &s, const float (&x)[VE]) {
    if constexpr (WIDE) {
      uint32_t o[kWords];
      pack<T, kWords>(x, o);
      char *p = reinterpret_cast<char *>(row + s.e);
      if constexpr (kWords % 4 == 0) {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) st16(p + 16 * i, o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
      } else {
        asm volatile("st.global.v2.b32 [%0], {%1,%2};" ::"l"(p), "r"(o[0]), "r"(o[1]) : "memory");
      }
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (s.e + i * s.cs < s.dim) row[s.e + i * s.cs] = El<T>::from(x[i]);
    }
  }
};
template <int VE, bool WIDE>
__device__ __forceinline__ Slice slice_of(int slab, int l, int G, int dim) {
  return WIDE ? Slice{(slab * G + l) * VE, 1, dim} : Slice{slab * G * VE + l, G, dim};
}
// log2 of the lanes that share a row of `dim` elements, VE each
inline int group_lg(int dim, int VE) {
  const int nvec = (dim + VE - 1) / VE;
  int lg = 0;
  while (lg < 5 && (1 << lg) < nvec) ++lg;
  return lg;
}
// Elements per lane: the narrower of the two types fills 16 bytes, or 8.
template <typename A, typename B>
constexpr int vec_of() {
  return 16 / (int)(sizeof(A) < sizeof(B) ? sizeof(A) : sizeof(B));
}
bool vec_ok(const void *p, int64_t stride, int dim, int ve, size_t es) {
  const size_t access = ve * es < 16 ? ve * es : 16;
  return dim % ve == 0 && reinterpret_cast<uintptr_t>(p) % access == 0 && (size_t)stride * es % access == 0;
}
constexpr int kLoose = 4;   // elements per lane of rows that are neither

// ---- lookup -----------------------------------------------------------------------------------------------------
struct EmbedArgs {
  const void *table, *ids;
  void *out;
  int32_t *flag;
  int64_t tokens, tstride, ostride, pad;
  int32_t rows, dim, ids64, lg;   // lg: log2 of the lanes that share a row
  float scale;
};

// A group of 2^lg lanes copies one row; a lane keeps kTok rows in flight.
template <typename T, typename TO, int VE, bool WIDE>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
  constexpr int kTok = 4;
  const int lane = threadIdx.x & 31, G = 1 << a.lg, l = lane & (G - 1);
  const int64_t per_warp = (int64_t)(32 >> a.lg);
  const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int64_t t0 = warp * per_warp * kTok + (lane >> a.lg);
  int64_t id[kTok];
#pragma unroll
  for (int j = 0; j < kTok; ++j) {
    const int64_t t = t0 + j * per_warp;
    id[j] = t < a.tokens ? load_id(a.ids, t, a.ids64) : -2;
    if (t < a.tokens && id[j] == a.pad) id[j] = -1;                         // zero row
    else if (t < a.tokens && (id[j] < 0 || id[j] >= a.rows)) id[j] = -3;    // no such row
  }
  bool bad = false;
  for (int slab = 0; slab * G * VE < a.dim; ++slab) {
    const Slice s = slice_of<VE, WIDE>(slab, l, G, a.dim);
    if (s.e >= a.dim) break;
    Elems<T, VE, WIDE> raw[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j)
      if (id[j] >= 0) raw[j].load(static_cast<const T *>(a.table) + id[j] * a.tstride, s);
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      if (id[j] != -2) {
        float x[VE];
        if (id[j] >= 0) {
          raw[j].get(x);
#pragma unroll
          for (int i = 0; i < VE; ++i) x[i] *= a.scale;
        } else {
          const float v = id[j] == -3 ? __int_as_float(0x7fffffff) : 0.f;
#pragma unroll
          for (int i = 0; i < VE; ++i) x[i] = v;
          bad |= id[j] == -3;
        }
        Elems<TO, VE, WIDE>::store(static_cast<TO *>(a.out) + (t0 + j * per_warp) * a.ostride, s, x);
      }
    }
  }
  if (bad && a.flag) *a.flag = 1;
}

template <typename T, typename TO, int VE, bool WIDE>
cudaError_t launch_embed(EmbedArgs a, cudaStream_t st) {
  a.lg = group_lg(a.dim, VE);
  const int64_t per_cta = (int64_t)(256 >> a.lg) * 4;
  const int64_t ctas = (a.tokens + per_cta - 1) / per_cta;
  if (ctas > 2147483647LL) return cudaErrorInvalidValue;
  embed_kernel<T, TO, VE, WIDE><<<(unsigned)ctas, 256, 0, st>>>(a);
  return cudaGetLastError();
}

template <typename T, typename TO>
cudaError_t dispatch_embed(const EmbedArgs &a, cudaStream_t st) {
  constexpr int VE = vec_of<T, TO>();
  auto fits = [&](int ve) {
    return vec_ok(a.table, a.tstride, a.dim, ve, sizeof(T)) && vec_ok(a.out, a.ostride, a.dim, ve, sizeof(TO));
  };
  if (fits(VE)) return launch_embed<T, TO, VE, true>(a, st);
  if (fits(VE / 2)) return launch_embed<T, TO, VE / 2, true>(a, st);
  return launch_embed<T, TO, kLoose, false>(a, st);
}

// ---- gradient ------------------------------------------------------------------------------------------------------
// The table to zero where no token adds to it.
struct Fill {
  char *base;             // null: nothing to zero (accumulation)
  int64_t row_bytes, stride_bytes, rows;
};
__device__ __forceinline__ void zero_bytes(char *p, int64_t n, int64_t i, int64_t step) {   // n and p: multiples of 2
  const uint32_t z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int64_t lead = min(n, (int64_t)((32u - (uint32_t)(reinterpret_cast<uintptr_t>(p) & 31u)) & 31u));
  const int64_t mid = (n - lead) >> 5, rest = n - lead - (mid << 5);
  char *const m = p + lead;
  int64_t q = i;
  for (; q + 3 * step < mid; q += 4 * step) {
    st32(m + (q << 5), z);
    st32(m + ((q + step) << 5), z);
    st32(m + ((q + 2 * step) << 5), z);
    st32(m + ((q + 3 * step) << 5), z);
  }
  for (; q < mid; q += step) st32(m + (q << 5), z);
  for (q = i; q < lead / 2; q += step) reinterpret_cast<uint16_t *>(p)[q] = 0;
  for (q = i; q < rest / 2; q += step) reinterpret_cast<uint16_t *>(m + (mid << 5))[q] = 0;
}
__device__ __forceinline__ void zero_table(const Fill &f, int cta, int ctas) {
  if (f.row_bytes == f.stride_bytes) {
    zero_bytes(f.base, f.row_bytes * f.rows, (int64_t)cta * blockDim.x + threadIdx.x, (int64_t)ctas * blockDim.x);
  } else {   // a warp per row
    const int warps = (int)(blockDim.x >> 5);
    for (int64_t r = (int64_t)cta * warps + (threadIdx.x >> 5); r < f.rows; r += (int64_t)ctas * warps)
      zero_bytes(f.base + r * f.stride_bytes, f.row_bytes, threadIdx.x & 31, 32);
  }
}

// The tokens' ids and what makes a sort key of them: the id, or `rows` (past every id) for padding and for ids that
// name no row.
struct Ids {
  const void *ids;
  int64_t tokens, pad;
  int32_t ids64, rows;
  int32_t *flag;
  __device__ __forceinline__ uint32_t key(int64_t t) const {
    const int64_t id = load_id(ids, t, ids64);
    const bool ok = id != pad && id >= 0 && id < rows;
    if (!ok && id != pad && flag) *flag = 1;
    return ok ? (uint32_t)id : (uint32_t)rows;
  }
};

// Ranks of a lane's items among the warp's items of the same digit in input order (item i of all lanes before item
// i + 1), through the warp's digit counters.  Lanes that hold the same digit are found from one ballot per digit bit,
// for all items side by side.
template <int ITEMS>
__device__ __forceinline__ void warp_ranks(uint16_t *counters, const uint32_t (&digit)[ITEMS], const bool (&ok)[ITEMS],
                                           int bits, int lane, uint32_t (&rank)[ITEMS]) {
  uint32_t peers[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    peers[i] = __ballot_sync(0xffffffffu, ok[i]);
    if (!ok[i]) peers[i] = ~peers[i];
  }
#pragma unroll 1
  for (int b = 0; b < bits; ++b) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t bal = __ballot_sync(0xffffffffu, (digit[i] >> b) & 1u);
      peers[i] &= ((digit[i] >> b) & 1u) ? bal : ~bal;
    }
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int leader = __ffs(peers[i]) - 1;
    uint32_t base = 0;
    if (lane == leader && ok[i]) {
      base = counters[digit[i]];
      counters[digit[i]] = (uint16_t)(base + __popc(peers[i]));
    }
    base = __shfl_sync(0xffffffffu, base, leader);
    __syncwarp();
    rank[i] = base + __popc(peers[i] & ((1u << lane) - 1u));
  }
}
// Exclusive scan of one value per thread (all threads of the block call it).
template <int NT>
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t *sh) {   // sh: NT / 32 words
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint32_t inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  if (lane == 31) sh[w] = inc;
  __syncthreads();
  const uint32_t before = __reduce_add_sync(0xffffffffu, lane < w ? sh[lane] : 0u);   // w <= NT / 32 words are read
  __syncthreads();
  return before + inc - v;
}

// ---- sort of up to 16 x 4096 tokens: one cluster, the items in its shared memory -----------------------------------
// Each CTA of the first cluster keeps its share of the items in registers; a pass ranks them (warp ballots, digit
// counters per warp, digit totals exchanged through distributed shared memory) and stores each to its place in the
// owning CTA's shared memory, the last pass to global memory.  The digit has up to 9 bits, so tables of fewer than
// 2^18 rows take two passes (the number of rows is itself a key).  Sorting on 16 SMs leaves the others idle, so the
// launch's other clusters zero the whole table (the rows that occur are written again by the sums).
constexpr int CS_THREADS = 1024, CS_WARPS = CS_THREADS / 32, CS_RADIX = 512;
template <int ITEMS>
constexpr size_t cs_smem() {
  return sizeof(uint64_t) * CS_THREADS * ITEMS + sizeof(uint16_t) * CS_WARPS * CS_RADIX + sizeof(uint32_t) * (2 * CS_RADIX + CS_WARPS);
}
template <int ITEMS>
__global__ void __launch_bounds__(CS_THREADS, 1)
cluster_sort_kernel(const Ids ids, int bits, uint64_t *out, const Fill fill) {
  constexpr uint32_t kPer = CS_THREADS * ITEMS;   // items of a CTA (the last one: what is left)
  constexpr int per = (int)kPer;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), b = (int)cluster.block_rank();
  if ((int)blockIdx.x >= C) {
    zero_table(fill, (int)blockIdx.x - C, (int)gridDim.x - C);
    return;
  }
  extern __shared__ __align__(16) unsigned char cs_dyn[];
  uint64_t *const buf = reinterpret_cast<uint64_t *>(cs_dyn);                        // [per]: key << 32 | position
  uint16_t(*const wc)[CS_RADIX] = reinterpret_cast<uint16_t(*)[CS_RADIX]>(buf + CS_THREADS * ITEMS);
  uint32_t *const hist = reinterpret_cast<uint32_t *>(wc + CS_WARPS);                // this CTA's digit totals
  uint32_t *const base = hist + CS_RADIX;                                            // first place of a digit's items of this CTA
  uint32_t *const sh = base + CS_RADIX;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int64_t n = ids.tokens;
  const int mine = (int)max((int64_t)0, min((int64_t)per, n - (int64_t)b * per));    // items of this CTA, always
  const int first = w * 32 * ITEMS + lane;                                           // place of this thread's item 0
  uint32_t key[ITEMS], pos[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int p = first + 32 * i;
    key[i] = 0;
    pos[i] = (uint32_t)(b * per + p);
    if (p < mine) key[i] = ids.key((int64_t)b * per + p);
  }
  const int passes = (bits + 8) / 9;
  int shift = 0;
  for (int pass = 0; pass < passes; ++pass) {
    const int db = (bits - shift + passes - pass - 1) / (passes - pass);   // bits of this digit
    const uint32_t mask = (1u << db) - 1u;
    for (int d = lane; d <= (int)mask; d += 32) wc[w][d] = 0;
    __syncwarp();
    uint32_t rank[ITEMS];
    constexpr int kSide = ITEMS < 4 ? ITEMS : 4;   // items ranked side by side
#pragma unroll
    for (int i = 0; i < ITEMS; i += kSide) {
      uint32_t dg[kSide], rk[kSide];
      bool ok[kSide];
#pragma unroll
      for (int j = 0; j < kSide; ++j) {
        dg[j] = (key[i + j] >> shift) & mask;
        ok[j] = first + 32 * (i + j) < mine;
      }
      warp_ranks<kSide>(wc[w], dg, ok, db, lane, rk);
#pragma unroll
      for (int j = 0; j < kSide; ++j) rank[i + j] = rk[j];
    }
    __syncthreads();
    if (tid <= (int)mask) {   // scan digit tid over the warps
      uint32_t run = 0;
#pragma unroll 8
      for (int q = 0; q < CS_WARPS; ++q) {
        const uint32_t v = wc[q][tid];
        wc[q][tid] = (uint16_t)run;
        run += v;
      }
      hist[tid] = run;
    }
    cluster.sync();   // digit totals of all CTAs; also: every CTA has taken its items out of its buffer
    uint32_t before = 0, total = 0;
    if (tid <= (int)mask) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {   // all in flight together
        const uint32_t v = q < C ? cluster.map_shared_rank(hist, q)[tid] : 0u;
        total += v;
        if (q < b) before += v;
      }
    }
    const uint32_t start = block_exclusive<CS_THREADS>(total, sh);
    if (tid <= (int)mask) base[tid] = start + before;
    __syncthreads();
    const bool last = pass + 1 == passes;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (first + 32 * i < mine) {
        const uint32_t d = (key[i] >> shift) & mask;
        const uint32_t to = base[d] + wc[w][d] + rank[i];
        const uint64_t item = (uint64_t)key[i] << 32 | pos[i];
        if (last) out[to] = item;
        else cluster.map_shared_rank(buf, to / kPer)[to % kPer] = item;
      }
    }
    cluster.sync();   // all items are in their places; also: nobody leaves while its totals may still be read
    if (!last) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int p = first + 32 * i;
        if (p < mine) {
          const uint64_t v = buf[p];
          key[i] = (uint32_t)(v >> 32);
          pos[i] = (uint32_t)v;
        }
      }
    }
    shift += db;
  }
}

// ---- sort of more tokens: two launches per digit of up to 10 bits -------------------------------------------------------
constexpr int LS_THREADS = 512, LS_WARPS = LS_THREADS / 32, LS_ITEMS = 8, LS_TILE = LS_THREADS * LS_ITEMS;
constexpr int LS_BITS = 10, LS_RADIX = 1 << LS_BITS;
constexpr int LS_BLOCKS = 296, LS_GROUP = 16, LS_GROUPS = (LS_BLOCKS + LS_GROUP - 1) / LS_GROUP;
static_assert(LS_RADIX <= 2 * LS_THREADS, "a thread scans two digits");
struct LargeSort {
  Ids ids;
  const uint64_t *in;             // key << 32 | position; null: from the ids
  uint64_t *out;
  uint32_t *hist;                 // [blocks][digits]
  uint32_t *group;                // [groups of LS_GROUP blocks][digits], zero before the histogram launch
  uint32_t *named;                // bit r: row r is named (marked by the last scatter), or null
  int64_t per_block;
  int32_t blocks, shift, bits;
};
__global__ void __launch_bounds__(LS_THREADS) large_hist_kernel(const LargeSort a) {
  __shared__ uint32_t h[LS_RADIX];
  const int digits = 1 << a.bits;
  const uint32_t mask = (uint32_t)digits - 1u;
  for (int d = threadIdx.x; d < digits; d += LS_THREADS) h[d] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.ids.tokens ? lo + a.per_block : a.ids.tokens;
#pragma unroll 4
  for (int64_t p = lo + threadIdx.x; p < hi; p += LS_THREADS)
    atomicAdd(&h[((a.in ? (uint32_t)(a.in[p] >> 32) : a.ids.key(p)) >> a.shift) & mask], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += LS_THREADS) {
    a.hist[blockIdx.x * digits + d] = h[d];
    if (h[d]) atomicAdd(&a.group[blockIdx.x / LS_GROUP * digits + d], h[d]);   // whole numbers: any order
  }
}
struct LargeMem {
  uint64_t stage[LS_TILE];
  uint16_t wc[LS_WARPS][LS_RADIX];
  uint32_t local[LS_RADIX], global[LS_RADIX];   // first staged place of a digit; its place in the output minus that
  uint32_t sh[LS_WARPS];
};
__global__ void __launch_bounds__(LS_THREADS, 2) large_scatter_kernel(const LargeSort a) {
  extern __shared__ __align__(16) unsigned char ls_dyn[];
  LargeMem &m = *reinterpret_cast<LargeMem *>(ls_dyn);
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, digits = 1 << a.bits;
  const uint32_t mask = (uint32_t)digits - 1u;
  const int64_t lo = blockIdx.x * a.per_block, hi = lo + a.per_block < a.ids.tokens ? lo + a.per_block : a.ids.tokens;
  uint64_t item[LS_ITEMS];
  auto fetch = [&](int64_t tile) {
#pragma unroll
    for (int i = 0; i < LS_ITEMS; ++i) {
      const int64_t p = tile + w * 32 * LS_ITEMS + lane + 32 * i;
      item[i] = p >= hi ? 0ull : a.in ? a.in[p] : (uint64_t)a.ids.key(p) << 32 | (uint32_t)p;
    }
  };
  fetch(lo);
  // where this block's items of digits 2 tid and 2 tid + 1 begin: all smaller digits, and the same digit of earlier
  // blocks, which are the earlier groups of blocks and the earlier blocks of the own group
  const bool scans = 2 * tid < digits;
  uint32_t run0 = 0, run1 = 0;
  {
    const int mygroup = (int)blockIdx.x / LS_GROUP, groups = (a.blocks + LS_GROUP - 1) / LS_GROUP;
    uint32_t b0 = 0, b1 = 0, t0 = 0, t1 = 0;
    if (scans) {
#pragma unroll
      for (int q = 0; q < LS_GROUPS; ++q) {
        if (q < groups) {
          const uint2 v = *reinterpret_cast<const uint2 *>(&a.group[q * digits + 2 * tid]);
          t0 += v.x;
          t1 += v.y;
          if (q < mygroup) {
            b0 += v.x;
            b1 += v.y;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < LS_GROUP; ++j) {
        const int q = mygroup * LS_GROUP + j;
        if (q < (int)blockIdx.x) {
          const uint2 v = *reinterpret_cast<const uint2 *>(&a.hist[q * digits + 2 * tid]);
          b0 += v.x;
          b1 += v.y;
        }
      }
    }
    const uint32_t first = block_exclusive<LS_THREADS>(t0 + t1, m.sh);
    run0 = first + b0;
    run1 = first + t0 + b1;
  }
  for (int64_t tile = lo; tile < hi; tile += LS_TILE) {
    for (int d = lane; d < digits; d += 32) m.wc[w][d] = 0;
    __syncwarp();
    uint32_t digit[LS_ITEMS], rank[LS_ITEMS];
    bool ok[LS_ITEMS];
#pragma unroll
    for (int i = 0; i < LS_ITEMS; ++i) {
      ok[i] = tile + w * 32 * LS_ITEMS + lane + 32 * i < hi;
      digit[i] = ((uint32_t)(item[i] >> 32) >> a.shift) & mask;
    }
    warp_ranks<LS_ITEMS>(m.wc[w], digit, ok, a.bits, lane, rank);
    __syncthreads();
    uint32_t c0 = 0, c1 = 0;
    if (scans) {   // two digits over the warps, as one word per warp
#pragma unroll
      for (int q = 0; q < LS_WARPS; ++q) {
        uint32_t *p = reinterpret_cast<uint32_t *>(&m.wc[q][2 * tid]);
        const uint32_t v = *p;
        *p = c0 | c1 << 16;
        c0 += v & 0xffffu;
        c1 += v >> 16;
      }
    }
    const uint32_t start = block_exclusive<LS_THREADS>(c0 + c1, m.sh);
    if (scans) {
      m.local[2 * tid] = start;
      m.local[2 * tid + 1] = start + c0;
      m.global[2 * tid] = run0 - start;
      m.global[2 * tid + 1] = run1 - (start + c0);
      run0 += c0;
      run1 += c1;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LS_ITEMS; ++i)
      if (ok[i]) m.stage[m.local[digit[i]] + m.wc[w][digit[i]] + rank[i]] = item[i];
    if (tile + LS_TILE < hi) fetch(tile + LS_TILE);
    __syncthreads();
    const int cn = (int)(hi - tile < LS_TILE ? hi - tile : LS_TILE);
    for (int i = tid; i < cn; i += LS_THREADS) {   // digit by digit, so that neighbouring threads write neighbouring places
      const uint64_t v = m.stage[i];
      const uint32_t key = (uint32_t)(v >> 32);
      a.out[m.global[(key >> a.shift) & mask] + (uint32_t)i] = v;
      // after the last digit a tile lies in key order, so each of its rows is marked once
      if (a.named && key < (uint32_t)a.ids.rows && (i == 0 || (uint32_t)(m.stage[i - 1] >> 32) != key))
        atomicOr(&a.named[key >> 5], 1u << (key & 31));
    }
    __syncthreads();
  }
}

struct SegArgs {
  const uint64_t *list;   // sorted: key << 32 | position
  const void *dy;
  void *dt;
  float *part;       // [ctas][2][dim]: sums that entered a CTA's range from the left, and that leave it to the right
  uint8_t *state;    // [ctas]: bit 0 = a run enters, bit 1 = that run also leaves (covers the range), bit 2 = a run starts here and leaves
  int64_t tokens, ystride, gstride;
  int32_t rows, dim, lg, run, accumulate;
  float scale;
  Ids ids;           // small batches: the tokens themselves, and the table to zero
  Fill fill;
  const uint32_t *named;   // bit r: some token names row r
  int32_t zero_ctas;       // the first CTAs zero the table
};

template <typename TO, int VE, bool WIDE>
__device__ __forceinline__ void write_row(const SegArgs &a, uint32_t key, const Slice &s, const float (&acc)[VE]) {
  TO *row = static_cast<TO *>(a.dt) + (int64_t)key * a.gstride;
  float o[VE];
  if (a.accumulate) {
    Elems<TO, VE, WIDE> old;
    old.load(row, s);
    old.get(o);
#pragma unroll
    for (int i = 0; i < VE; ++i) o[i] = fmaf(acc[i], a.scale, o[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) o[i] = acc[i] * a.scale;
  }
  Elems<TO, VE, WIDE>::store(row, s, o);
}
// a CTA's partial row
template <int VE>
__device__ __forceinline__ void write_part(float *row, const Slice &s, const float (&acc)[VE]) {
#pragma unroll
  for (int i = 0; i < VE; ++i)
    if (s.e + i * s.cs < s.dim) row[s.e + i * s.cs] = acc[i];
}

// Zeroes rows [r0, r0 + n) of the table where `named` (bit i: row r0 + i) is 0.  Rows of whole 32-byte words take one
// store per lane and word, others go by zero_bytes.
__device__ __forceinline__ void zero_unnamed(const Fill &f, int64_t r0, int64_t n, const uint32_t *named) {
  constexpr int kRows = 4;   // rows a group of lanes has in flight
  int lg = 0;                // lanes per row
  while (lg < 5 && (32 << lg) < f.row_bytes) ++lg;
  const int per = 256 >> lg, l = (int)threadIdx.x & ((1 << lg) - 1);
  const bool whole = ((reinterpret_cast<uintptr_t>(f.base) | (uintptr_t)f.row_bytes | (uintptr_t)f.stride_bytes) & 31u) == 0;
  const uint32_t z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int64_t i0 = (int64_t)threadIdx.x >> lg; i0 < n; i0 += kRows * per) {
    uint32_t word[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int64_t i = i0 + j * per;
      word[j] = i < n ? named[i >> 5] >> (i & 31) & 1u : 1u;
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (word[j]) continue;
      char *row = f.base + (r0 + i0 + j * per) * f.stride_bytes;
      if (whole) {
        for (int q = l; q < (int)(f.row_bytes >> 5); q += 1 << lg) st32(row + (q << 5), z);
      } else {
        zero_bytes(row, f.row_bytes, l, 1 << lg);
      }
    }
  }
}
// This CTA's share of the rows that no token names, so that every row of the table is written once and the zeroing
// runs beside the sums.  In a small batch the named rows are marked here, from the tokens; else the sort marked them.
constexpr int kSmallTokens = 256, kSmallRows = 1 << 24, kMarkRows = 4096;
template <bool SMALL>
__device__ __forceinline__ void zero_others(const SegArgs &a, int cta, int ctas) {
  // shares in whole words of marks
  const int64_t words = ((int64_t)a.rows + 31) / 32;
  const int64_t lo = words * cta / ctas * 32, hi = min((int64_t)a.rows, words * (cta + 1) / ctas * 32);
  if (!SMALL) {
    if (lo < hi) zero_unnamed(a.fill, lo, hi - lo, a.named + lo / 32);
    return;
  }
  __shared__ uint32_t named[kMarkRows / 32];
  for (int64_t r0 = lo; r0 < hi; r0 += kMarkRows) {
    const int n = (int)(hi - r0 < kMarkRows ? hi - r0 : kMarkRows);
    for (int i = threadIdx.x; i < (n + 31) / 32; i += 256) named[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < (int)a.tokens; i += 256) {
      const int64_t r = (int64_t)a.ids.key(i) - r0;
      if (r >= 0 && r < n) atomicOr(&named[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    zero_unnamed(a.fill, r0, n, named);
    __syncthreads();
  }
}

// CTA x, y: places [x * per, (x + 1) * per) of the sorted list, per = groups * run; columns of slab y.  Dynamic shared
// memory: the keys and positions of those places.
template <typename T, typename TO, int VE, bool WIDE, bool SMALL>
__global__ void __launch_bounds__(256, 3) embed_seg_kernel(const SegArgs a) {
  constexpr int kFly = Elems<T, VE, WIDE>::kWords > 4 ? 4 : 8;   // rows a lane keeps in flight
  if ((int)blockIdx.x < a.zero_ctas) {   // the first ones, so that they run beside the sums
    zero_others<SMALL>(a, (int)(blockIdx.x * gridDim.y + blockIdx.y), a.zero_ctas * (int)gridDim.y);
    return;
  }
  const int cta = (int)blockIdx.x - a.zero_ctas;
  __shared__ float head[256][VE], tail[256][VE];
  __shared__ uint8_t gstate[256];   // per group, as SegArgs::state
  __shared__ uint32_t cta_state, key_before, key_after;
  extern __shared__ __align__(16) uint32_t places[];
  const int G = 1 << a.lg, ng = 256 >> a.lg, g = threadIdx.x >> a.lg, l = threadIdx.x & (G - 1);
  const Slice slice = slice_of<VE, WIDE>((int)blockIdx.y, l, G, a.dim);
  const bool col = slice.e < a.dim;
  const int per = ng * a.run;
  const int64_t c0 = (int64_t)cta * per;
  const int cn = (int)(a.tokens - c0 < per ? a.tokens - c0 : per);   // places of this CTA
  uint32_t *const skey = places, *const spos = places + per;
  const uint32_t none = (uint32_t)a.rows;
  if (threadIdx.x == 0) cta_state = 0;
  if constexpr (SMALL) {   // all tokens are here: sorted by counting, key and position in one word (rows < 2^24)
    uint32_t *const word = spos + per;
    for (int i = threadIdx.x; i < ((cn + 3) & ~3); i += 256)
      word[i] = i < cn ? a.ids.key(i) << 8 | (uint32_t)i : 0xffffffffu;
    if (threadIdx.x == 0) key_before = key_after = 0xffffffffu;
    __syncthreads();
    for (int i = threadIdx.x; i < cn; i += 256) {
      const uint32_t mine = word[i];
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < cn; j += 4) {
        const uint4 o = *reinterpret_cast<const uint4 *>(&word[j]);
        place += (o.x < mine) + (o.y < mine) + (o.z < mine) + (o.w < mine);
      }
      skey[place] = mine >> 8;
      spos[place] = mine & 255u;
    }
  } else {
    for (int i = threadIdx.x; i < cn; i += 256) {
      const uint64_t v = a.list[c0 + i];
      skey[i] = (uint32_t)(v >> 32);
      spos[i] = (uint32_t)v;
    }
    if (threadIdx.x == 0) {
      key_before = c0 > 0 ? (uint32_t)(a.list[c0 - 1] >> 32) : 0xffffffffu;
      key_after = c0 + cn < a.tokens ? (uint32_t)(a.list[c0 + cn] >> 32) : 0xffffffffu;
    }
  }
  __syncthreads();
  const int b = min(g * a.run, cn), end = min(b + a.run, cn);
  uint32_t st = 0;
  if (b < end) {
    uint32_t cur = skey[b];
    bool entered = (b > 0 ? skey[b - 1] : key_before) == cur;   // the run began before this group's range
    const bool leaves = (end < cn ? skey[end] : key_after) == skey[end - 1];
    float acc[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) acc[i] = 0.f;
    auto flush = [&]() {
      if (cur != none && col) {
        if (entered) {
#pragma unroll
          for (int i = 0; i < VE; ++i) head[threadIdx.x][i] = acc[i];
        } else {
          write_row<TO, VE, WIDE>(a, cur, slice, acc);
        }
      }
      if (entered && cur != none) st |= 1;
#pragma unroll
      for (int i = 0; i < VE; ++i) acc[i] = 0.f;
      entered = false;
    };
    const T *const dy = static_cast<const T *>(a.dy);
#pragma unroll 1
    for (int p = b; p < end; p += kFly) {
      Elems<T, VE, WIDE> x[kFly];
#pragma unroll
      for (int j = 0; j < kFly; ++j)
        if (p + j < end && skey[p + j] != none && col) x[j].load(dy + (int64_t)spos[p + j] * a.ystride, slice);
#pragma unroll
      for (int j = 0; j < kFly; ++j) {
        if (p + j < end) {
          const uint32_t k = skey[p + j];
          if (k != cur) {
            flush();
            cur = k;
          }
          if (k != none && col) {
            float v[VE];
            x[j].get(v);
#pragma unroll
            for (int i = 0; i < VE; ++i) acc[i] += v[i];
          }
        }
      }
    }
    if (!leaves || cur == none) {
      flush();
    } else if (entered) {   // covers the whole range
      if (col) {
#pragma unroll
        for (int i = 0; i < VE; ++i) head[threadIdx.x][i] = acc[i];
      }
      st |= 3;
    } else {
      if (col) {
#pragma unroll
        for (int i = 0; i < VE; ++i) tail[threadIdx.x][i] = acc[i];
      }
      st |= 4;
    }
  }
  if (l == 0) gstate[g] = (uint8_t)st;
  __syncthreads();

  // runs that cross group borders: the group where such a run starts (or group 0, for the run that enters the
  // CTA) adds the pieces up in group order
  uint32_t crossing = 0;
  for (int pass = 0; pass < 2; ++pass) {
    const bool enter = pass == 0;
    if (enter ? (g != 0 || !(gstate[0] & 1)) : !(gstate[g] & 4)) continue;
    float acc[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) acc[i] = enter ? 0.f : tail[threadIdx.x][i];
    int q = enter ? 0 : g + 1;
    bool open = true;   // the run reaches group q
    for (; q < ng && open; ++q) {
      if (!(gstate[q] & 1)) { open = q * a.run >= cn; break; }
#pragma unroll
      for (int i = 0; i < VE; ++i) acc[i] += head[q * G + l][i];
      open = gstate[q] & 2;
    }
    if (enter) {
      crossing |= 1 | (open ? 2 : 0);
      if (col) write_part<VE>(a.part + ((int64_t)cta * 2) * a.dim, slice, acc);
    } else if (open) {
      crossing |= 4;
      if (col) write_part<VE>(a.part + ((int64_t)cta * 2 + 1) * a.dim, slice, acc);
    } else if (col) {
      write_row<TO, VE, WIDE>(a, skey[(g + 1) * a.run], slice, acc);
    }
  }
  // bits 0 and 1 come from group 0, bit 2 from the one group whose run leaves the CTA
  if (l == 0 && crossing) atomicOr(&cta_state, crossing);
  __syncthreads();
  if (!SMALL && threadIdx.x == 0 && blockIdx.y == 0) a.state[cta] = (uint8_t)cta_state;   // (a small batch is one range and has no workspace)
}

// One CTA per list range whose last run leaves it: that run's partial rows, in order.  The rows are dealt to the
// warps in contiguous shares and the shares are added in warp order.
template <typename TO>
__global__ void __launch_bounds__(256) embed_join_kernel(const SegArgs a, int64_t per, int32_t ctas) {
  const int32_t c = blockIdx.x;
  if (!(a.state[c] & 4)) return;
  __shared__ int32_t last_s;
  __shared__ float share[8][128];
  // last range the run reaches: the first after c that it does not cover
  if (threadIdx.x == 0) last_s = ctas - 1;
  __syncthreads();
  for (int32_t q0 = c + 1; q0 < ctas; q0 += 256) {
    const int32_t q = q0 + (int32_t)threadIdx.x;
    const bool stop = q < ctas && !(a.state[q] & 2);
    if (stop) atomicMin(&last_s, q);
    if (__syncthreads_or(stop)) break;
  }
  const uint32_t key = (uint32_t)(a.list[(int64_t)(c + 1) * per] >> 32);
  const int n = last_s - c;   // entering rows of ranges c + 1 .. last
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int q0 = (int)((int64_t)n * w / 8), q1 = (int)((int64_t)n * (w + 1) / 8);
  for (int e0 = 0; e0 < a.dim; e0 += 128) {   // four columns a lane
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const float *row = a.part + ((int64_t)(c + 1 + q0) * 2) * a.dim + e0 + lane;
#pragma unroll 4
    for (int q = q0; q < q1; ++q, row += 2 * (int64_t)a.dim) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e0 + 32 * j + lane < a.dim) acc[j] += row[32 * j];
    }
    const bool mine = threadIdx.x < 128 && e0 + (int)threadIdx.x < a.dim;   // thread t: column e0 + t
    float v = mine ? a.part[((int64_t)c * 2 + 1) * a.dim + e0 + threadIdx.x] : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) share[w][32 * j + lane] = acc[j];
    __syncthreads();
    if (mine) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v += share[q][threadIdx.x];
      const float o[1] = {v};
      write_row<TO, 1, false>(a, key, Slice{e0 + (int)threadIdx.x, 1, a.dim}, o);
    }
    __syncthreads();
  }
}

constexpr int32_t kDimMax = 1 << 20;   // the column slabs are the grid's second dimension

// Places a group of lanes sums in registers (fewest and most), and the most places of a CTA.  At least 4: 5,000 x 128 bf16
// 15.3 us, with 8 16.0, with 16 17.8.  At most 32: 1M x 128 bf16 185 us, with 16 195 (more partial rows to join).
constexpr int kRunMin = 4, kRun = 32, kPlaces = 2048;
// Places per group when 2^lg lanes share a row: one CTA when that is enough (nothing to join), else runs as long as still
// give every SM two CTAs.
inline int run_of(int64_t tokens, int lg) {
  const int ng = 256 >> lg, most = kPlaces / ng < kRun ? kPlaces / ng : kRun;
  const int64_t want = tokens <= (int64_t)ng * most ? (tokens + ng - 1) / ng : tokens / ((int64_t)ng * 2 * kSMs);
  return (int)(want < kRunMin ? kRunMin : want > most ? most : want);
}

template <typename T, typename TO, int VE, bool WIDE>
cudaError_t launch_seg(SegArgs a, cudaStream_t st) {
  const int nvec = (a.dim + VE - 1) / VE;
  a.lg = group_lg(a.dim, VE);
  const int ng = 256 >> a.lg;
  a.run = run_of(a.tokens, a.lg);
  const int64_t per = (int64_t)ng * a.run;
  const int64_t ctas = (a.tokens + per - 1) / per;
  const int slabs = (nvec + (1 << a.lg) - 1) >> a.lg;
  if (slabs > 65535) return cudaErrorInvalidValue;
  // zeroing CTAs: one per 32 KB, at most a resident wave of them
  const int64_t zero = a.fill.base ? a.fill.row_bytes * a.fill.rows : 0;
  int64_t nf = (zero + 32767) / 32768;
  if (nf > 2 * kSMs) nf = 2 * kSMs;
  a.zero_ctas = (int32_t)((nf + slabs - 1) / slabs);
  if (!a.list) {   // small batch: one launch sorts, sums and zeroes
    embed_seg_kernel<T, TO, VE, WIDE, true><<<dim3((unsigned)(1 + a.zero_ctas), (unsigned)slabs), 256, (size_t)(3 * per + 4) * 4, st>>>(a);
    return cudaGetLastError();
  }
  embed_seg_kernel<T, TO, VE, WIDE, false><<<dim3((unsigned)(ctas + a.zero_ctas), (unsigned)slabs), 256, (size_t)per * 8, st>>>(a);
  CK(cudaGetLastError());
  if (ctas > 1) {
    embed_join_kernel<TO><<<(unsigned)(ctas - 1), 256, 0, st>>>(a, per, (int32_t)ctas);
    CK(cudaGetLastError());
  }
  return cudaSuccess;
}

template <typename T, typename TO>
cudaError_t dispatch_seg(const SegArgs &a, cudaStream_t st) {
  constexpr int VE = vec_of<T, TO>();
  auto fits = [&](int ve) {
    return vec_ok(a.dy, a.ystride, a.dim, ve, sizeof(T)) && vec_ok(a.dt, a.gstride, a.dim, ve, sizeof(TO));
  };
  if (fits(VE)) return launch_seg<T, TO, VE, true>(a, st);
  if (fits(VE / 2)) return launch_seg<T, TO, VE / 2, true>(a, st);
  return launch_seg<T, TO, kLoose, false>(a, st);
}

template <typename T>
cudaError_t dispatch_seg_out(const SegArgs &a, int out_dt, cudaStream_t st) {
  if (out_dt == TSID_DT_F32) return dispatch_seg<T, float>(a, st);
  if (out_dt == TSID_DT_BF16) return dispatch_seg<T, __nv_bfloat16>(a, st);
  return dispatch_seg<T, __half>(a, st);
}

template <typename T>
cudaError_t dispatch_embed_out(const EmbedArgs &a, int out_dt, cudaStream_t st) {
  if (out_dt == TSID_DT_F32) return dispatch_embed<T, float>(a, st);
  if (out_dt == TSID_DT_BF16) return dispatch_embed<T, __nv_bfloat16>(a, st);
  return dispatch_embed<T, __half>(a, st);
}

struct GradCarve {
  uint64_t *A, *B;
  uint32_t *hist, *group, *named;
  float *part;
  uint8_t *state;
  size_t bytes;
};
// A batch that one CTA of the sums covers (8 groups of 32 lanes with 32 places each) is sorted there (65 x 64 bf16: 4.5 us
// in one launch, 10.1 with a sort of its own; 256 x 64: 6.1 and 10.7).
static_assert(kSmallTokens <= 8 * kRun && kSmallTokens <= kPlaces, "one CTA per slab");
inline bool small_batch(int64_t tokens, int32_t rows) { return tokens <= kSmallTokens && rows < kSmallRows; }
// most tokens of the one-cluster sort (100,000 tokens: 51 us there with 16 items a thread, 31 us by the large sort)
constexpr int64_t kClusterTokens = 16 * 4 * CS_THREADS;
GradCarve carve_grad(void *base, int64_t tokens, int32_t rows, int32_t dim) {
  Carver cv(base);
  GradCarve c = {};
  if (small_batch(tokens, rows)) return c;
  const size_t nt = (size_t)tokens + 1;
  size_t ctas = 0;   // of the sums, for any alignment of the rows, hence any number of lanes that share one
  for (int lg = 0; lg <= 5; ++lg) ctas = std::max(ctas, nt / ((size_t)(256 >> lg) * run_of(tokens, lg)) + 1);
  c.A = cv.take<uint64_t>(nt);
  if (tokens > kClusterTokens) {
    c.B = cv.take<uint64_t>(nt);
    c.hist = cv.take<uint32_t>((size_t)LS_RADIX * LS_BLOCKS);
    c.group = cv.take<uint32_t>((size_t)LS_RADIX * LS_GROUPS * 4 + ((size_t)rows + 31) / 32);
    c.named = c.group + (size_t)LS_RADIX * LS_GROUPS * 4;
  }
  c.part = cv.take<float>(ctas * 2 * (size_t)dim);
  c.state = cv.take<uint8_t>(ctas);
  c.bytes = cv.off;
  return c;
}

template <int ITEMS>
cudaError_t launch_cluster_sort(const Ids &ids, int bits, const GradCarve &c, const Fill &fill, cudaStream_t st) {
  auto kern = cluster_sort_kernel<ITEMS>;
  CK(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  CK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cs_smem<ITEMS>()));
  const int64_t cap = (int64_t)CS_THREADS * ITEMS;
  const int C = (int)((ids.tokens + cap - 1) / cap);
  // zeroing CTAs: one per 64 KB, at most what is left of the SMs, in whole clusters
  const int64_t zero = fill.base ? fill.rows * fill.row_bytes : 0;
  int64_t nf = (zero + 65535) / 65536;
  if (nf > kSMs - C) nf = kSMs - C;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(C * (1 + (nf + C - 1) / C)));
  cfg.blockDim = dim3(CS_THREADS);
  cfg.dynamicSmemBytes = cs_smem<ITEMS>();
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, ids, bits, c.A, fill);
}

// Sorts the tokens by key; *list receives the sorted list.  The one-cluster sort also zeroes the table (and clears
// `fill`), the large one marks the rows that are named.
cudaError_t sort_tokens(const Ids &ids, const GradCarve &c, Fill &fill, cudaStream_t st, const uint64_t **list) {
  const int bits = bits_for((uint32_t)ids.rows);
  if (ids.tokens <= kClusterTokens) {
    *list = c.A;
    // as few items a thread as 16 CTAs allow (whole gradient, 16,000 tokens: 18.1 us with one, 23.0 with four; 3,000: 15.5
    // and 19.4; 32,000: 23.6 with two, 27.5 with four)
    if (ids.tokens <= 16 * CS_THREADS) CK(launch_cluster_sort<1>(ids, bits, c, fill, st));
    else if (ids.tokens <= 32 * CS_THREADS) CK(launch_cluster_sort<2>(ids, bits, c, fill, st));
    else CK(launch_cluster_sort<4>(ids, bits, c, fill, st));
    fill.base = nullptr;
    return cudaSuccess;
  }
  const bool mark = fill.base != nullptr;
  CK(cudaFuncSetAttribute(large_scatter_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LargeMem)));
  const int passes = (bits + LS_BITS - 1) / LS_BITS;
  const int64_t tiles = (ids.tokens + LS_TILE - 1) / LS_TILE;
  const int blocks = (int)(tiles < LS_BLOCKS ? tiles : LS_BLOCKS);
  LargeSort a = {ids, nullptr, c.A, c.hist, c.group, nullptr,
                 (tiles + blocks - 1) / blocks * LS_TILE, blocks, 0, 0};
  // the group totals and the marks lie side by side
  CK(cudaMemsetAsync(c.group, 0, sizeof(uint32_t) * (LS_RADIX * LS_GROUPS * 4 + (mark ? ((size_t)ids.rows + 31) / 32 : 0)), st));
  for (int p = 0; p < passes; ++p) {
    a.group = c.group + (size_t)p * LS_RADIX * LS_GROUPS;
    a.bits = (bits - a.shift + passes - p - 1) / (passes - p);
    if (p + 1 == passes && mark) a.named = c.named;
    large_hist_kernel<<<(unsigned)blocks, LS_THREADS, 0, st>>>(a);
    large_scatter_kernel<<<(unsigned)blocks, LS_THREADS, sizeof(LargeMem), st>>>(a);
    CK(cudaGetLastError());
    a.shift += a.bits;
    a.in = a.out;
    a.out = a.out == c.A ? c.B : c.A;
  }
  *list = a.in;
  return cudaSuccess;
}

bool aligned_to(const void *p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; }

}  // namespace
}  // namespace tsid

using namespace tsid;

extern "C" {

tsid_status_t tsid_embed(int64_t n_tokens, int32_t n_rows, int32_t dim, const void *d_table, int32_t table_dtype,
                         int64_t table_stride, const void *d_ids, int32_t ids_i64, int64_t pad_id, float scale,
                         void *d_out, int32_t out_dtype, int64_t out_stride, int32_t *d_flag_or_null, void *stream) {
  if (n_tokens < 0 || n_rows < 1 || dim < 1) return refuse(TSID_ERR_INVALID_ARG, "n_tokens must be >= 0, n_rows and dim >= 1");
  if (dim > kRowMax) return refuse(TSID_ERR_UNSUPPORTED, "dim above 2^31 - 1024");
  if (!dtype_ok(table_dtype) || !dtype_ok(out_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad dtype");
  if (n_tokens == 0) return TSID_OK;
  if (n_tokens > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
  if (!d_table || !d_ids || !d_out) return refuse(TSID_ERR_INVALID_ARG, "table, ids or out is null");
  if (!aligned_to(d_table, dtype_bytes(table_dtype)) || !aligned_to(d_out, dtype_bytes(out_dtype)) ||
      !aligned_to(d_ids, ids_i64 ? 8 : 4))
    return refuse(TSID_ERR_INVALID_ARG, "table, ids or out is not aligned to its elements");
  if ((n_rows > 1 && table_stride < dim) || (n_tokens > 1 && out_stride < dim))
    return refuse(TSID_ERR_INVALID_ARG, "a row stride is smaller than dim");
  EmbedArgs a = {d_table, d_ids, d_out, d_flag_or_null, n_tokens, table_stride, out_stride, pad_id, n_rows, dim,
                 ids_i64, 0, scale};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = table_dtype == TSID_DT_F32    ? dispatch_embed_out<float>(a, out_dtype, st)
                  : table_dtype == TSID_DT_BF16 ? dispatch_embed_out<__nv_bfloat16>(a, out_dtype, st)
                                                : dispatch_embed_out<__half>(a, out_dtype, st);
  return e == cudaSuccess ? TSID_OK : refuse(TSID_ERR_CUDA, cudaGetErrorString(e));
}

tsid_status_t tsid_embed_grad_workspace_bytes(int64_t n_tokens, int32_t n_rows, int32_t dim, size_t *h_bytes_out) {
  if (!h_bytes_out || n_tokens < 0 || n_rows < 1 || dim < 1)
    return refuse(TSID_ERR_INVALID_ARG, "n_tokens must be >= 0, n_rows and dim >= 1");
  if (n_tokens > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
  *h_bytes_out = carve_grad(nullptr, n_tokens, n_rows, dim).bytes;
  return TSID_OK;
}

tsid_status_t tsid_embed_grad(int64_t n_tokens, int32_t n_rows, int32_t dim, const void *d_grad_out,
                              int32_t grad_out_dtype, int64_t grad_out_stride, const void *d_ids, int32_t ids_i64,
                              int64_t pad_id, float scale, void *d_grad_table, int32_t grad_table_dtype,
                              int64_t grad_table_stride, int32_t accumulate, void *workspace, size_t workspace_bytes,
                              int32_t *d_flag_or_null, void *stream) {
  if (n_tokens < 0 || n_rows < 1 || dim < 1) return refuse(TSID_ERR_INVALID_ARG, "n_tokens must be >= 0, n_rows and dim >= 1");
  if (dim > kDimMax) return refuse(TSID_ERR_UNSUPPORTED, "dim above 2^20");
  if (!dtype_ok(grad_out_dtype) || !dtype_ok(grad_table_dtype)) return refuse(TSID_ERR_INVALID_ARG, "bad dtype");
  if (n_tokens > 2147483647LL) return refuse(TSID_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
  if (!d_grad_table || (n_tokens > 0 && (!d_grad_out || !d_ids))) return refuse(TSID_ERR_INVALID_ARG, "grad_out, ids or grad_table is null");
  if (!aligned_to(d_grad_out, dtype_bytes(grad_out_dtype)) || !aligned_to(d_grad_table, dtype_bytes(grad_table_dtype)) ||
      !aligned_to(d_ids, ids_i64 ? 8 : 4))
    return refuse(TSID_ERR_INVALID_ARG, "grad_out, ids or grad_table is not aligned to its elements");
  if ((n_rows > 1 && grad_table_stride < dim) || (n_tokens > 1 && grad_out_stride < dim))
    return refuse(TSID_ERR_INVALID_ARG, "a row stride is smaller than dim");
  GradCarve c = carve_grad(workspace, n_tokens, n_rows, dim);
  if (c.bytes > 0) {
    if (!workspace || !aligned_to(workspace, 256)) return refuse(TSID_ERR_INVALID_ARG, "workspace is null or not 256-byte aligned");
    if (workspace_bytes < c.bytes) return refuse(TSID_ERR_OOM, "workspace smaller than tsid_embed_grad_workspace_bytes");
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto run = [&]() -> cudaError_t {
    const size_t es = dtype_bytes(grad_table_dtype);
    const size_t row = (size_t)dim * es;
    if (n_tokens == 0) {
      if (accumulate) return cudaSuccess;
      if (grad_table_stride == dim || n_rows == 1) return cudaMemsetAsync(d_grad_table, 0, row * n_rows, st);
      return cudaMemset2DAsync(d_grad_table, (size_t)grad_table_stride * es, 0, row, (size_t)n_rows, st);
    }
    Fill fill = {};
    if (!accumulate) fill = {static_cast<char *>(d_grad_table), (int64_t)row, grad_table_stride * (int64_t)es, n_rows};
    SegArgs a = {};
    a.ids = {d_ids, n_tokens, pad_id, ids_i64, n_rows, d_flag_or_null};
    a.fill = fill;
    a.dy = d_grad_out;
    a.dt = d_grad_table;
    a.part = c.part;
    a.state = c.state;
    a.tokens = n_tokens;
    a.ystride = grad_out_stride;
    a.gstride = grad_table_stride;
    a.rows = n_rows;
    a.dim = dim;
    a.accumulate = accumulate;
    a.scale = scale;
    if (!small_batch(n_tokens, n_rows)) CK(sort_tokens(a.ids, c, a.fill, st, &a.list));
    a.named = c.named;
    if (grad_out_dtype == TSID_DT_F32) return dispatch_seg_out<float>(a, grad_table_dtype, st);
    if (grad_out_dtype == TSID_DT_BF16) return dispatch_seg_out<__nv_bfloat16>(a, grad_table_dtype, st);
    return dispatch_seg_out<__half>(a, grad_table_dtype, st);
  };
  cudaError_t e = run();
  return e == cudaSuccess ? TSID_OK : refuse(TSID_ERR_CUDA, cudaGetErrorString(e));
}

}  // extern "C"
