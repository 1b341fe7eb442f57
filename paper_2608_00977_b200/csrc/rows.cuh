// Shared pieces of the kernels that stream rows of scores or factor rows (embed.cu, token_logprobs.cu,
// distill.cu): element types, 16-byte chunks of a row at any alignment, packed fp32 arithmetic, the running
// maximum and sums of a softmax, and the order in which columns are ranked.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tsid_internal.cuh"

namespace tsid {

// ---- element types -----------------------------------------------------------------------------------------
template <typename T>
struct El;
template <>
struct El<float> {
  static constexpr int kPer16 = 4;                     // elements of a 16-byte chunk
  static constexpr uint32_t kFill = 0xff800000u;       // word of minus infinities
  static constexpr int kShift = 0;                     // low bits of the fp32 pattern that are always equal
  static __device__ __forceinline__ float load(const float *p) { return *p; }
  static __device__ __forceinline__ float from(float v) { return v; }
};
template <>
struct El<__nv_bfloat16> {
  static constexpr int kPer16 = 8;
  static constexpr uint32_t kFill = 0xff80ff80u;
  static constexpr int kShift = 16;
  static __device__ __forceinline__ float load(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct El<__half> {
  static constexpr int kPer16 = 8;
  static constexpr uint32_t kFill = 0xfc00fc00u;
  static constexpr int kShift = 13;
  static __device__ __forceinline__ float load(const __half *p) { return __half2float(*p); }
  static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
};

inline size_t dtype_bytes(int dt) { return dt == TSID_DT_F32 ? 4 : 2; }
inline bool dtype_ok(int dt) { return dt == TSID_DT_F32 || dt == TSID_DT_BF16 || dt == TSID_DT_F16; }

// two floats of a word of 16-bit elements (exact)
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
// one rounding to nearest even: the only one between the fp32 result and the stored element
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// the elements of NW words as floats, and back
template <typename T, int NW>
__device__ __forceinline__ void unpack(const uint32_t (&w)[NW], float *x) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < NW; ++i) x[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float2 v = unpack2<T>(w[i]);
      x[2 * i] = v.x;
      x[2 * i + 1] = v.y;
    }
  }
}
template <typename T, int NW>
__device__ __forceinline__ void pack(const float *x, uint32_t (&w)[NW]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = __float_as_uint(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
  }
}

// ---- a row as 16-byte chunks ----------------------------------------------------------------------------------------
// A row of V elements may start at any element boundary.  It is cut at the 16-byte boundaries of the address
// space: chunk c holds the elements [c h - lead, (c + 1) h - lead), h = elements per chunk, lead = elements between
// the boundary below the row's start and the start.  Every chunk but the first and the last is one aligned load;
// those two are read element by element, inside the row only.
//
// A lane works on a pair of chunks 32 apart, so that the 32 lanes of a warp read 512 consecutive bytes at a time:
// pair p = (p >> 5, lane) is the chunks c = 64 (p >> 5) + lane and c + 32.  (A lane that took 32 consecutive bytes
// by two 16-byte accesses would fetch every 32-byte sector twice.)
template <typename T>
struct RowChunks {
  static constexpr int h = El<T>::kPer16;
  const T *row;
  int32_t V, lead, pairs;   // pairs: a multiple of 32
  int32_t w0, wn;           // pairs [w0, w0 + wn) have two whole chunks: all groups of 32 pairs but the first and the last
  __device__ __forceinline__ RowChunks(const T *r, int32_t v) : row(r), V(v) {
    lead = (int32_t)((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(T));
    const int64_t chunks = ((int64_t)lead + v + h - 1) / h;
    pairs = (int32_t)((chunks + 63) / 64 * 32);
    w0 = lead > 0 ? 32 : 0;
    const int32_t w1 = (int32_t)(((int64_t)lead + v) / (64 * h) * 32);   // groups that end inside the row
    wn = w1 > w0 ? w1 - w0 : 0;
  }
  static __device__ __forceinline__ int32_t chunk(int32_t p) { return 2 * p - (p & 31); }
  __device__ __forceinline__ int64_t first(int32_t c) const { return (int64_t)c * h - lead; }
  __device__ __forceinline__ bool whole(int32_t c) const {
    const int64_t e0 = first(c);
    return e0 >= 0 && e0 + h <= V;
  }
  __device__ __forceinline__ bool whole_pair(int32_t p) const { return (uint32_t)(p - w0) < (uint32_t)wn; }
};

// the words of chunk c into w[at .. at + 3]; elements outside the row read as minus infinity
template <typename T>
__device__ __forceinline__ void load_chunk_slow(const RowChunks<T> &r, int32_t c, uint32_t (&w)[8], int at) {
  const int64_t e0 = r.first(c);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t v;
    if constexpr (sizeof(T) == 4) {
      const int64_t e = e0 + i;
      v = e >= 0 && e < r.V ? reinterpret_cast<const volatile uint32_t *>(r.row)[e] : El<T>::kFill;
    } else {
      const volatile uint16_t *p = reinterpret_cast<const volatile uint16_t *>(r.row);
      const int64_t e = e0 + 2 * i;
      const uint32_t lo = e >= 0 && e < r.V ? p[e] : (El<T>::kFill & 0xffffu);
      const uint32_t hi = e + 1 >= 0 && e + 1 < r.V ? p[e + 1] : (El<T>::kFill & 0xffffu);
      v = lo | (hi << 16);
    }
    if (at == 0) w[i] = v;
    else w[4 + i] = v;
  }
}
__device__ __forceinline__ void ld16(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d, const void *p) {
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "l"(p));
}
__device__ __forceinline__ void st16(void *p, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.global.v4.b32 [%4], {%0,%1,%2,%3};" ::"r"(a), "r"(b), "r"(c), "r"(d), "l"(p) : "memory");
}
__device__ __forceinline__ void st32(void *p, const uint32_t (&w)[8]) {   // 32-byte aligned
  asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p)
               : "memory");
}
// the words of both chunks of pair p: w[0..3] the first, w[4..7] the one 32 chunks on
template <typename T>
__device__ __forceinline__ void load_pair(const RowChunks<T> &r, int32_t p, uint32_t (&w)[8]) {
  const int32_t c = r.chunk(p);
  if (r.whole_pair(p)) {
    const char *q = reinterpret_cast<const char *>(r.row + r.first(c));
    ld16(w[0], w[1], w[2], w[3], q);
    ld16(w[4], w[5], w[6], w[7], q + 512);
  } else {
    load_chunk_slow(r, c, w, 0);
    load_chunk_slow(r, c + 32, w, 4);
  }
}
// element i of a pair's 2 h elements lies at column at(i) (which may be outside the row in a chunk that is not whole)
template <typename T>
struct PairColumns {
  int64_t a, b;
  __device__ __forceinline__ PairColumns(const RowChunks<T> &r, int32_t p) : a(r.first(r.chunk(p))), b(a + 32 * RowChunks<T>::h) {}
  __device__ __forceinline__ int64_t at(int i) const { return i < RowChunks<T>::h ? a + i : b + (i - RowChunks<T>::h); }
};

// Whether the chunks of the input row are 16-byte aligned in an output row that starts at `out`.
template <typename T, typename TO>
__device__ __forceinline__ bool wide_rows(const RowChunks<T> &r, const TO *out) {
  return ((reinterpret_cast<uintptr_t>(out) + sizeof(TO) * (size_t)(RowChunks<T>::h - r.lead)) & 15u) == 0;
}
// largest element of four words (NaN is passed over); 16-bit elements are compared two at a time
template <typename T>
__device__ __forceinline__ float chunk_max(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(a), __uint_as_float(b)), fmaxf(__uint_as_float(c), __uint_as_float(d)));
  } else if constexpr (El<T>::kShift == 16) {
    typedef const __nv_bfloat162 *P;
    const __nv_bfloat162 m = __hmax2(__hmax2(*P(&a), *P(&b)), __hmax2(*P(&c), *P(&d)));
    return fmaxf(__low2float(m), __high2float(m));
  } else {
    typedef const __half2 *P;
    const __half2 m = __hmax2(__hmax2(*P(&a), *P(&b)), __hmax2(*P(&c), *P(&d)));
    return fmaxf(__low2float(m), __high2float(m));
  }
}

// ---- a thread's pairs through shared memory -----------------------------------------------------------------------
// A thread copies its own pairs into its own slots with asynchronous 16-byte copies, kStages - 1 pairs ahead of the
// arithmetic, and reads them back itself: nothing is synchronised between threads, and the loads in flight cost
// no registers.  The two chunks of a pair lie in two planes, so neighbouring threads use neighbouring words.
constexpr int kStages = 3;
template <int NT>
struct PairRing {
  uint4 slot[kStages][2][NT];
};
template <typename T, int NT>
struct PairStream {
  static constexpr int kStep = NT * 32;   // bytes from a thread's pair to its next one, in the row and in the ring
  const RowChunks<T> &r;
  const char *src;      // the thread's next pair to copy
  int32_t p, end;       // its number, and the end of the CTA's part
  uint32_t base, fill;  // ring, and place of the next copy
  __device__ __forceinline__ PairStream(const RowChunks<T> &rb, PairRing<NT> &ring, int32_t p0, int32_t p1)
      : r(rb), src(reinterpret_cast<const char *>(rb.row) + rb.first(rb.chunk(p0)) * (int64_t)sizeof(T)), p(p0), end(p1),
        base((uint32_t)__cvta_generic_to_shared(&ring.slot[0][0][threadIdx.x])), fill(base) {
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) issue();
  }
  __device__ __forceinline__ void issue() {
    if (p < end && r.whole_pair(p)) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(fill), "l"(src) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(fill + NT * 16), "l"(src + 512) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");   // one group per pair, also for those read directly
    p += NT;
    src += kStep;
    fill = fill == base + (kStages - 1) * kStep ? base : fill + kStep;
  }
  // calls f(pair, words) for the thread's pairs in turn; before that, patch(pair, slot) may change the pair in its slot
  // (the first chunk's shared address; the second lies NT * 16 bytes on)
  template <typename F, typename P>
  __device__ __forceinline__ void run(F f, P patch) {
    uint32_t from = base;
    for (int32_t q = p - (kStages - 1) * NT; q < end; q += NT) {
      issue();
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      uint32_t w[8];
      if (!r.whole_pair(q)) {
        load_pair(r, q, w);
        asm volatile("st.shared.v4.b32 [%4], {%0,%1,%2,%3};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(from) : "memory");
        asm volatile("st.shared.v4.b32 [%4], {%0,%1,%2,%3};" ::"r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(from + NT * 16) : "memory");
      }
      patch(q, from);
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory");
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(from + NT * 16) : "memory");
      from = from == base + (kStages - 1) * kStep ? base : from + kStep;
      f(q, w);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  template <typename F>
  __device__ __forceinline__ void run(F f) {
    run(f, [](int32_t, uint32_t) {});
  }
};

// ---- elementwise passes from one row to another ------------------------------------------------------------------------
// Pairs p0, p0 + step, ... of a thread, read kAhead of them ahead and written to the same columns of another row: x of
// f(pair, x) comes in as the elements and leaves as the results.  Addresses move by constant strides.
template <typename T, typename TO, int kAhead>
struct PairMap {
  static constexpr int h = RowChunks<T>::h;
  const RowChunks<T> &r;
  TO *out;
  bool wide;
  const char *src;   // the thread's next pair to read
  char *dst;         // the next one to write
  int32_t p, step;
  uint32_t raw[kAhead][8];
  __device__ __forceinline__ PairMap(const RowChunks<T> &rb, TO *o, int32_t p0, int32_t st)
      : r(rb), out(o), wide(wide_rows(rb, o)), src(reinterpret_cast<const char *>(rb.row + rb.first(rb.chunk(p0)))),
        dst(reinterpret_cast<char *>(o + rb.first(rb.chunk(p0)))), p(p0), step(st) {}
  __device__ __forceinline__ void fetch(int32_t q, int32_t end, uint32_t (&w)[8]) {
    if (q < end) {
      if (r.whole_pair(q)) {
        ld16(w[0], w[1], w[2], w[3], src);
        ld16(w[4], w[5], w[6], w[7], src + 512);
      } else {
        load_pair(r, q, w);
      }
    }
    src += (int64_t)step * 32;
  }
  __device__ __forceinline__ void start(int32_t end) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(p + i * step, end, raw[i]);
  }
  template <typename F, typename G>
  __device__ __forceinline__ void run(int32_t end, F f, G after) {
    for (int32_t q0 = p; q0 < end; q0 += kAhead * step) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int32_t q = q0 + i * step;
        if (q < end) {
          float x[2 * h];
          unpack<T, 8>(raw[i], x);
          fetch(q + kAhead * step, end, raw[i]);
          f(q, x);
          if (wide && r.whole_pair(q)) {
            constexpr int nw = 2 * h * (int)sizeof(TO) / 4, half = h * (int)sizeof(TO);   // bytes of a chunk's results
            uint32_t o[nw];
            pack<TO, nw>(x, o);
#pragma unroll
            for (int j = 0; j < nw / 2; j += 4) {
              st16(dst + 4 * j, o[j], o[j + 1], o[j + 2], o[j + 3]);
              st16(dst + 32 * half + 4 * j, o[nw / 2 + j], o[nw / 2 + j + 1], o[nw / 2 + j + 2], o[nw / 2 + j + 3]);
            }
          } else {
            const PairColumns<T> col(r, q);
#pragma unroll
            for (int j = 0; j < 2 * h; ++j) {
              const int64_t e = col.at(j);
              if (e >= 0 && e < r.V) out[e] = El<TO>::from(x[j]);
            }
          }
          after(q);
        }
        dst += (int64_t)step * 32 * (int)(sizeof(TO) / sizeof(T) ? sizeof(TO) / sizeof(T) : 1);
      }
    }
  }
};

// ---- packed fp32 arithmetic (two lanes per instruction) ------------------------------------------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 mk2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void un2(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

constexpr float kLowest = -3.402823466e38f;   // reference point of a row that has shown no finite element yet
constexpr float kFloor2 = -200.f;             // 2^-200 is zero in fp32: exponents below need not be told apart
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kScaleMin = 1e-20f, kScaleMax = 1e20f;   // accepted scales: c and kFloor2 / c stay far inside fp32

// scale (x - m) of finite scores as far apart as the type allows: the difference is taken in halves, which is exact, so
// it cannot overflow before a small scale brings it back into range
__device__ __forceinline__ float half_diff(float x, float m) { return 0.5f * x - 0.5f * m; }
__device__ __forceinline__ float scaled_diff(float x, float m, float scale) { return half_diff(x, m) * scale * 2.f; }

// ---- running sums of a softmax -------------------------------------------------------------------------------------
// Of the elements seen so far, with c = scale / log 2 and a reference m:
//   s = sum 2^t,   u = sum 2^t t,   t = c (x - m).
// Excluded elements (minus infinity) add exact zeros; NaN and plus infinity make s a NaN, which no later element removes.
struct Soft {
  float m, s, u;
};
// maximum over the warp of floats that are not NaN
__device__ __forceinline__ float warp_max(float x);
// the warp's parts about their common maximum, added up by a fixed tree; all lanes hold the same bits
__device__ __forceinline__ Soft soft_warp(Soft v, float c) {
  Soft r;
  r.m = warp_max(v.m);
  const float d = fmaxf((v.m - r.m) * c, kFloor2), f = ex2(d);
  r.u = f * fmaf(v.s, d, v.u);
  r.s = f * v.s;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
    r.u += __shfl_xor_sync(0xffffffffu, r.u, o);
  }
  return r;
}

// A thread's running sums over the elements of its pairs (U: whether u is wanted).
//
// The reference moves only when an element exceeds it by more than kSlack in the exponent: sums of terms up to 2^16
// have the same relative accuracy, and a reference that followed the maximum would make some lane of nearly every
// warp rescale at nearly every step.
//
// t is one multiply-add, t = c x - (c m) with the rounded product.  The product's rounding error, which is the same
// for all terms, is known exactly (delta = fma(c, m, -(c m))) and taken out of the sums when the reference moves and at
// the end.  Every term carries the factor 2^delta until then, so delta has to stay small: it is at most half a unit of
// c m, 2^-5 while |c m| < 2^20, but hundreds from |c m| = 2^33 (scores of 1e10 at scale 1), which is beyond fp32's exponents.
// From 2^20 on, t = c (x - m) in two steps, which has no such term (one instruction more per two elements).
constexpr float kSlack = 16.f;
constexpr float kProductMax = 1048576.f;
template <int N, bool U>
struct RunningSoft {
  float c, slack, m, delta, high;
  bool far;          // |c m| has reached kProductMax: t in two steps
  f32x2 c2, negmc;   // minus the rounded product
  f32x2 s2, u2;
  __device__ __forceinline__ explicit RunningSoft(float scale)
      : c(scale * kLog2e), slack(kSlack / (scale * kLog2e)), m(kLowest), delta(0.f), high(-INFINITY), far(true),
        c2(mk2(c, c)), negmc(mk2(0.f, 0.f)), s2(mk2(0.f, 0.f)), u2(s2) {}
  // cm: the largest of x, or anything between it and a value not far above
  __device__ __forceinline__ void take(const float (&x)[N], float cm) {
    if (cm > high) {
      const float m1 = fmaxf(cm, kLowest), mc = m1 * c;
      far = !(fabsf(mc) < kProductMax);
      const float delta1 = far ? 0.f : fmaf(m1, c, -mc);
      const float d = fmaxf(fmaf(m - m1, c, delta1 - delta), kFloor2), f = ex2(d);
      const f32x2 f2 = mk2(f, f);
      if (U) u2 = mul2(f2, fma2(s2, mk2(d, d), u2));
      s2 = mul2(s2, f2);
      m = m1;
      delta = delta1;
      high = m1 + slack;
      negmc = mk2(-mc, -mc);
    }
    if (!far) {
#pragma unroll
      for (int i = 0; i < N; i += 2) add(fma2(mk2(x[i], x[i + 1]), c2, negmc));
    } else {
      const f32x2 negm = mk2(-m, -m);
#pragma unroll
      for (int i = 0; i < N; i += 2) add(mul2(add2(mk2(x[i], x[i + 1]), negm), c2));
    }
  }
  __device__ __forceinline__ void add(f32x2 t) {
    float t0, t1;
    un2(t, t0, t1);
    if (U) {   // an excluded element: zero times the floor, not zero times minus infinity
      t0 = max_nan(t0, kFloor2);
      t1 = max_nan(t1, kFloor2);
    }
    const f32x2 e = mk2(ex2(t0), ex2(t1));
    s2 = add2(s2, e);
    if (U) u2 = fma2(e, mk2(t0, t1), u2);
  }
  // The sums about `top`, the largest of the elements (minus infinity: there were none).  Dividing by its own term, as
  // the pass formed it, leaves exactly 1 of it and takes delta out of the others, so s >= 1 and a row with nearly all its
  // mass in one column keeps what the others add.
  __device__ __forceinline__ Soft result(float top) const {
    float a, b, tm;
    Soft r;
    un2(s2, a, b);
    r.m = kLowest;
    r.s = a + b;
    r.u = 0.f;
    if (top > -INFINITY) {
      un2(negmc, tm, tm);
      tm = far ? (top - m) * c : fmaf(top, c, tm);
      const float e = ex2(tm), s = r.s;
      r.m = top;
      r.s = s / e;
      if (U) {
        un2(u2, a, b);
        r.u = fmaf(-tm, s, a + b) / e;
      }
    }
    return r;
  }
};

// ---- ranking order ------------------------------------------------------------------------------------------------
// Whole-number image of a float that sorts like the float; minus zero and zero are one value.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float order_inv(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

__device__ __forceinline__ float warp_max(float x) {
  return order_inv(__reduce_max_sync(0xffffffffu, order_of(x)));
}

// Block-wide lower bound of the k-th largest of distinct keys (0 = no key): the threads' keys are counted into 256
// equal bins of the range [lo, hi] that holds at least k of them, the bin that the k-th falls into is found from
// the top, and the search goes on inside that bin while more than `enough` keys lie at or above its lower edge.
// One round is a shared-memory histogram and one warp's scan, and on ordinary data one round is all there is.
// Returns a bound with k <= #{keys >= bound}, <= enough unless a single key value is left.
struct KeyHist {
  uint32_t bin[256];
  uint32_t found, above;
};
template <int NT, int NK>
__device__ __forceinline__ uint64_t kth_bound(const uint64_t (&key)[NK], uint64_t lo, uint64_t hi, int k, int enough,
                                              KeyHist &h) {
  uint32_t above = 0;   // keys above hi
  for (;;) {
    const uint64_t range = hi - lo;
    const int sh = max(0, 56 - __clzll((long long)(range | 1)));   // the range's top 8 bits are the bin
    for (int i = threadIdx.x; i < 256; i += NT) h.bin[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NK; ++i)
      if (key[i] >= lo && key[i] <= hi && key[i] != 0) atomicAdd(&h.bin[(uint32_t)((key[i] - lo) >> sh)], 1u);
    __syncthreads();
    if (threadIdx.x < 32) {
      const int top = 255 - 8 * (int)threadIdx.x;   // this lane's bins: top, top - 1, ..., top - 7
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += c[j] = h.bin[top - j];
      uint32_t inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o);
        if ((int)threadIdx.x >= o) inc += u;
      }
      uint32_t run = above + inc - sum;
      if (run < (uint32_t)k && run + sum >= (uint32_t)k) {
        int j = 0;
        while (run + c[0] < (uint32_t)k) {   // rotate, so that the registers are indexed by constants
          run += c[0];
#pragma unroll
          for (int q = 0; q < 7; ++q) c[q] = c[q + 1];
          ++j;
        }
        h.found = (uint32_t)(top - j);
        h.above = run;
        h.bin[0] = run + c[0];   // keys at or above the bin's lower edge
      }
    }
    __syncthreads();
    const uint32_t bin = h.found, at_least = h.bin[0];
    const uint64_t edge = lo + ((uint64_t)bin << sh);
    if (at_least <= (uint32_t)enough || sh == 0) return edge;
    above = h.above;
    const uint64_t end = edge + ((1ull << sh) - 1);
    hi = end < hi ? end : hi;
    lo = edge;
    __syncthreads();
  }
}

// The largest number of CTAs that share one row (a thread-block cluster; above 8 needs the opt-in).
constexpr int kRowClusterMax = 16;
constexpr int kSMs = 148;

// Reports a refused call: the message tsid_last_error(NULL) returns, and the status.
tsid_status_t refuse(tsid_status_t st, const char *msg);

}  // namespace tsid
