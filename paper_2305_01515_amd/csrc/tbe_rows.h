// Shared by the operators on rows (norm, short convolution, selective scan): packs at any address, parameters of any type, small
// functions, sums of partial results.
#pragma once
#include <algorithm>
#include <initializer_list>

#include "tbe_dense.h"

namespace tbe {

// Memory of a call: `rows` pieces of `row` bytes, `stride` apart (0: all the same one)
struct Span {
  const void *p;
  int64_t row, stride, rows;
};
inline Span span(const void *p, int64_t bytes) { return {p, bytes, bytes, 1}; }
inline Span span(const void *p, int64_t elems, int64_t stride, int64_t rows, int bytes) { return {p, elems * bytes, stride * bytes, rows}; }
inline bool same_span(const Span &a, const Span &b) { return a.p == b.p && a.row == b.row && (a.stride == b.stride || (a.rows <= 1 && b.rows <= 1)) && a.rows == b.rows; }

// Whether two have a byte in common.  Of rows that lie apart by two different strides it is not found out: columns of one piece of memory may be meant.
inline bool overlap(Span a, Span b) {
  for (Span *s : {&a, &b}) {
    if (!s->p || s->row <= 0 || s->rows <= 0) return false;
    if (s->rows > 1 && s->stride == s->row) s->row *= s->rows, s->rows = 1;
    if (s->rows == 1 || s->stride == 0) s->stride = s->row, s->rows = 1;
  }
  const int64_t at = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);  // of b from a's first byte
  if (at >= (a.rows - 1) * a.stride + a.row || at + (b.rows - 1) * b.stride + b.row <= 0) return false;
  if (b.rows == 1) {
    // the first row of a that ends behind b's first byte
    const int64_t i = at < a.row ? 0 : (at - a.row) / a.stride + 1;
    return i < a.rows && i * a.stride < at + b.row;
  }
  if (a.rows == 1) return overlap(b, a);
  if (a.stride != b.stride) return false;
  int64_t k = at / a.stride, rest = at % a.stride;  // b's first row begins `rest` bytes behind where a's row k does
  if (rest < 0) --k, rest += a.stride;
  auto meet = [&](int64_t k) { return k < a.rows && k + b.rows > 0; };  // some row j of b and row j + k of a are both there
  return (rest < a.row && meet(k)) || (rest + b.row > a.stride && meet(k + 1));
}
inline int check_apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span &w : written)
    for (const Span &r : read)
      if (overlap(w, r)) return report(TBE_EINVAL, "what the call writes overlaps what it reads");
  return TBE_OK;
}

// V elements (the first `n` of them, if fewer) at any address that an element may have, as fp32; what is beyond n reads as zero
template <class E, int V>
__device__ inline void load_floats(const E *p, int n, float (&to)[V]) {
  if (n >= V) {
    E r[V];
    __builtin_memcpy(r, p, sizeof r);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = (float)r[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = i < n ? (float)p[i] : 0.0f;
  }
}
template <class E, int V>
__device__ inline void store_floats(E *p, int n, const float (&from)[V]) {
  if (n >= V) {
    Pack<E, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.e[i] = (E)from[i];
    __builtin_memcpy(p, &r, sizeof r);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (E)from[i];
  }
}

// V elements as they lie in memory.  (As elements, each of 16 bits would have a register of its own.)
template <class E, int V> struct alignas(sizeof(E) * V) Words {
  uint32_t w[sizeof(E) * V / 4];
  __device__ float get(int i) const {
    if constexpr (sizeof(E) == 4) {
      return __builtin_bit_cast(float, w[i]);
    } else {
      const uint16_t b = (uint16_t)(w[i / 2] >> (i % 2 * 16));
      return (float)__builtin_bit_cast(E, b);
    }
  }
};
// the first n of them, if fewer: zero beyond
template <class E, int V>
__device__ inline void load_words(const E *p, int n, Words<E, V> &to) {
  if (n >= V) {
    __builtin_memcpy(to.w, p, sizeof to.w);
  } else {
#pragma unroll
    for (unsigned i = 0; i < sizeof to.w / 4; ++i) to.w[i] = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i >= n) continue;
      if constexpr (sizeof(E) == 4) to.w[i] = ((const uint32_t *)p)[i];
      else to.w[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (i % 2 * 16);
    }
  }
}

template <class E, int V>
__device__ inline void store_words(E *p, int n, const Words<E, V> &from) {
  if (n >= V) {
    __builtin_memcpy(p, from.w, sizeof from.w);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i >= n) continue;
      if constexpr (sizeof(E) == 4) ((uint32_t *)p)[i] = from.w[i];
      else ((uint16_t *)p)[i] = (uint16_t)(from.w[i / 2] >> (i % 2 * 16));
    }
  }
}

// quotient of numbers that mostly have 32 bits
__device__ inline int64_t quotient(int64_t a, int64_t b) { return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }

// parameters of a type that is known at run time only
__device__ inline float load_param(const void *p, int dtype, int64_t i) {
  return dtype == TBE_FP32 ? ((const float *)p)[i] : dtype == TBE_FP16 ? (float)((const _Float16 *)p)[i] : (float)((const __bf16 *)p)[i];
}
template <int V>
__device__ inline void load_params(const void *p, int dtype, int64_t at, int n, float (&to)[V]) {
  if (dtype == TBE_FP32) load_floats<float, V>((const float *)p + at, n, to);
  else if (dtype == TBE_FP16) load_floats<_Float16, V>((const _Float16 *)p + at, n, to);
  else load_floats<__bf16, V>((const __bf16 *)p + at, n, to);
}

// how many of the ascending offsets[0 .. n) are at most `row`, the same in all lanes of a wavefront: 64 places are looked at at once
__device__ inline int64_t count_up_to(const int64_t *off, int64_t n, int64_t row) {
  int64_t lo = 0, hi = n;  // off[i] <= row for i < lo, not for i >= hi
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + (int64_t)(threadIdx.x & 63) * step;
    const int c = __popcll(__ballot(at < hi && off[at] <= row));  // the first c places are
    if (c == 0) return lo;
    lo += (int64_t)(c - 1) * step + 1;
    hi = min(hi, lo + step - 1);
  }
  return lo;
}

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// The exponential is the hardware's power of two of the rounded v log2(e): the rounding is up to |v| 2^-24 of the exponential, log2(e) in 32 bits 0.22 |v| 2^-24, so
// a sigmoid is off by up to (1.25 |v| + 8) 2^-24 of itself (silu: 65.2 x 2^-24 at most, measured); below -87 it is zero.
__device__ inline float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -kLog2e)); }

// Sums over the parts of [parts][n] fp32 numbers, in a fixed order: 32 columns a workgroup, 32 lanes a column with every 32nd part each.
// A row of `width` columns has `cut` columns that go to `to`, one that goes to `next`, one that goes to `other` (each unless null).
constexpr int kSumColumns = 32;
__global__ __launch_bounds__(1024) static void sum_parts_kernel(const float *parts, int64_t count, int64_t n, int width, int cut, float *to, float *next,
                                                                float *other) {
  __shared__ float lds[32][kSumColumns + 1];
  const int c = threadIdx.x % kSumColumns, s = threadIdx.x / kSumColumns;
  const int64_t at = (int64_t)blockIdx.x * kSumColumns + c;
  float v = 0.0f;
  if (at < n) {
#pragma unroll 8
    for (int64_t p = s; p < count; p += 32) v += parts[p * n + at];
  }
  lds[s][c] = v;
  for (int half = 16; half >= 1; half /= 2) {
    __syncthreads();
    if (s < half) lds[s][c] += lds[s + half][c];
  }
  if (s == 0 && at < n) {
    const int64_t r = at / width;
    const int k = (int)(at % width);
    float *p = k < cut ? to : k == cut ? next : other;
    if (p) p[k < cut ? r * cut + k : r] = lds[0][c];
  }
}

inline int64_t divide_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline void sum_parts(const float *parts, int64_t count, int64_t n, int width, int cut, float *to, float *next, float *other, hipStream_t st) {
  sum_parts_kernel<<<dim3((unsigned)divide_up(n, kSumColumns)), dim3(1024), 0, st>>>(parts, count, n, width, cut, to, next, other);
}

// waits for the stream; what its kernels have reported in *d_err since the last look, which is cleared
inline int check_errors(int32_t *d_err, hipStream_t st) {
  int32_t err = 0;
  hipError_t e = hipMemcpyAsync(&err, d_err, sizeof err, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e == hipSuccess && err) {
    e = hipMemsetAsync(d_err, 0, sizeof err, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
  }
  if (e != hipSuccess) return report_hip(e);
  if (err == 1) return report(TBE_EINVAL, "offsets that do not ascend from 0 to the number of rows");
  if (err == 2) return report(TBE_ERANGE, "a slot is not below the number of states");
  return TBE_OK;
}

}  // namespace tbe
