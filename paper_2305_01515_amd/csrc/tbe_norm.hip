// Root-mean-square norm of rows with the residual's addition in front: forward, results in 8 bits with scales, backward.
// Contract: include/tbe.h.
//
//   s = x + residual, stored in the residual's type; the norm is that of the stored row, so the backward that reads it finds the same.
//   out = s rstd w, rstd = 1 / sqrt(mean(s s) + eps);
//   with d = dout w:  ds = rstd (d - s rstd mean(d s rstd)) + what comes from the next layers,  dw = sum over rows of dout s rstd.
//
// Bound by memory: each row is read once, into registers.  A row lies on lanes of V elements (16 bytes of x) a pack, P packs a lane:
// a part of a wavefront or a whole one (ROW_THREADS 64), or a workgroup of ROW_THREADS lanes.  245760 rows of 128 in bfloat16 with an fp32 residual:
// forward 64 us (5.9 TB/s, more than a copy of 1 GB, 5.2: rows of this size stay in the last-level cache in part), backward 97 us (5.2 TB/s); 16384 rows of 4096 to 8 bits 95 us (5.0 TB/s; with 32 elements a lane instead of 16, half of
// them beyond the row, 134 us of vector instructions).  The backward of long rows has few wavefronts a SIMD (two for 8192 elements), and beyond that reads its inputs
// twice: 8192 rows of 8192 in bfloat16 147 us (2.7 TB/s), 4096 of 16384 210 (1.9), in fp32 163 (4.9) and 286 (2.8).
#include <algorithm>
#include <new>
#include <type_traits>

#include "tbe_rows.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostParts = 1024;          // workgroups of the backward, each with a partial sum of dw
constexpr int64_t kPartFloats = 1ll << 24;    // ... of so many numbers together

template <class E> constexpr int kPack = 16 / sizeof(E);

struct NormArgs {
  const void *x, *residual, *weight;
  int64_t xs, rs, rows, row0;
  int dim, lanes, weight_dtype;
  float eps;
  void *out, *summed;
  int64_t os, ss;
  float *rstd, *scales;
  int group, groups;  // elements that share a scale, scales of a row
};

// sum over the lanes of a row, the same in all of them
template <int ROW_THREADS>
__device__ inline float row_sum(float v, int lanes, float *lds) {
  for (int o = 1; o < (ROW_THREADS > 64 ? 64 : lanes); o *= 2) v += __shfl_xor(v, o);
  if constexpr (ROW_THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < ROW_THREADS / 64; ++i) v += lds[i];
  }
  return v;
}
// largest of non-negative numbers by their bits: a NaN is larger than any number
template <int ROW_THREADS>
__device__ inline uint32_t row_max(uint32_t v, int lanes, uint32_t *lds) {
  for (int o = 1; o < (ROW_THREADS > 64 ? 64 : lanes); o *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  if constexpr (ROW_THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < ROW_THREADS / 64; ++i) v = max(v, lds[i]);
  }
  return v;
}

// Codes of V numbers whose group has the largest magnitude `top`, as 448ths of it.  Where the scale is zero (`zero`), so are the codes.  A
// group with an infinity or a NaN has such a scale, and codes of NaN.  A code is the even one of two where 448 v / top lies half way between them, which
// happens: rows and weights of 16 bits have few products (2 in 10000 codes of bfloat16).  So the quotient is found to its last bit: what is left of 448 v behind
// the first quotient times top is found exactly, and divided once more.
template <int V>
__device__ inline void store_codes(uint8_t *p, int n, const float (&v)[V], float top, bool zero) {
  uint32_t w[V / 4];
  auto codes = [&](float up) {
    const float t = top * up, r = t > 0.0f ? 1.0f / t : 0.0f, f = 448.0f * r;
    auto quotient = [&](float v) {
      const float x = v * up, q = x * f, p = q * t;
      return __builtin_fmaf(__builtin_fmaf(x, 448.0f, -p) - __builtin_fmaf(q, t, -p), r, q);
    };
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[i]), quotient(v[i + 1]), 0, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[i + 2]), quotient(v[i + 3]), c, true);
      w[i / 4] = (uint32_t)c;
    }
  };
  // (one over a very small number would be infinite, 448 of a very large one too)
  if (top < 0x1p-100f || top > 0x1p100f) codes(top < 1.0f ? 0x1p100f : 0x1p-100f);
  else codes(1.0f);
  if (zero) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = 0;
  }
  if (n >= V) {
    __builtin_memcpy(p, w, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (uint8_t)(w[i / 4] >> (i % 4 * 8));
  }
}

// R: the residual's type (void: there is none); BITS8: the results are codes
template <class E, class R, bool BITS8, int ROW_THREADS, int P>
__global__ __launch_bounds__(ROW_THREADS > 64 ? ROW_THREADS : kThreads) void norm_kernel(NormArgs a) {
  constexpr int V = kPack<E>;
  constexpr bool RES = !__is_same(R, void);
  using S = std::conditional_t<RES, R, E>;
  __shared__ float lds[ROW_THREADS > 64 ? ROW_THREADS / 64 : 1];
  const int L = ROW_THREADS > 64 ? ROW_THREADS : a.lanes, lane = threadIdx.x & (L - 1);
  int64_t row = a.row0 + (ROW_THREADS > 64 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L);
  const bool there = row < a.rows;
  if (!there) row = a.rows - 1;  // its lanes exchange like the others' and store nothing
  const E *x = (const E *)a.x + row * a.xs;
  float v[P][V], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (lane + i * L) * V;
    load_floats<E, V>(x + at, a.dim - at, v[i]);
    if constexpr (RES) {
      float o[V];
      load_floats<S, V>((const S *)a.residual + row * a.rs + at, a.dim - at, o);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = (float)(S)(v[i][j] + o[j]);
    }
  }
  // the row has been read whole, by the lane that writes there, so the sum may lie where x or the residual do
  if constexpr (RES) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      if (there) store_floats<S, V>((S *)a.summed + row * a.ss + at, a.dim - at, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) sum += v[i][j] * v[i][j];
  sum = row_sum<ROW_THREADS>(sum, L, lds);
  const float rstd = 1.0f / sqrtf(sum / (float)a.dim + a.eps);
  if (there && lane == 0 && a.rstd) a.rstd[row] = rstd;
  // Codes do not depend on rstd but for their scale: they are found from s w times the power of two in rstd, which rounds nothing.
  const float power = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, rstd) & 0x7F800000u), times = BITS8 ? power : rstd;
  const float rest = power > 0.0f ? rstd / power : 1.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (lane + i * L) * V;
    float w[V];
    load_params<V>(a.weight, a.weight_dtype, at, a.dim - at, w);
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * times * w[j];
    if (at + V > a.dim) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = at + j < a.dim ? v[i][j] : 0.0f;  // (an infinite rstd has no part beyond the row)
    }
  }
  if constexpr (!BITS8) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      if (there) store_floats<E, V>((E *)a.out + row * a.os + at, a.dim - at, v[i]);
    }
  } else {
    uint32_t top[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      top[i] = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) top[i] = max(top[i], __builtin_bit_cast(uint32_t, fabsf(v[i][j])));
    }
    if (a.groups == 1) {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < P; ++i) t = max(t, top[i]);
      t = row_max<ROW_THREADS>(t, L, (uint32_t *)lds);
#pragma unroll
      for (int i = 0; i < P; ++i) top[i] = t;
    } else {  // lanes side by side share a scale
#pragma unroll
      for (int i = 0; i < P; ++i)
        for (int k = 1; k < a.group / V; k *= 2) top[i] = max(top[i], (uint32_t)__shfl_xor((int)top[i], k));
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      const float t = __builtin_bit_cast(float, top[i]);
      if (!there || at >= a.dim) continue;
      const float scale = t * rest / 448.0f;
      if (at % a.group == 0) a.scales[row * a.groups + at / a.group] = scale;
      store_codes<V>((uint8_t *)a.out + row * a.os + at, a.dim - at, v[i], t, scale == 0.0f);
    }
  }
}

struct NormGrad {
  const void *s, *dout, *ds, *weight;   // the stored sum, gradients of the result and (or null) of the stored sum
  int64_t ss, dos, dss, rows;
  int dim, lanes, weight_dtype;
  const float *rstd;
  void *dx, *dres;                      // either may be null
  int64_t dxs, drs;
  float *parts;                         // [workgroups][dim], or null
};

// E: type of x, the result and dx; S: of the stored sum, its gradient and dres.  A workgroup takes every gridDim-th group of rows and keeps its sum of dw.
template <class E, class S, int ROW_THREADS, int P>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormGrad a) {
  constexpr int V = kPack<E>;
  __shared__ float lds[4];
  extern __shared__ float sums[];  // rows on parts of wavefronts: [kThreads / L][L V P] sums of dw
  const int L = ROW_THREADS > 64 ? ROW_THREADS : a.lanes, lane = threadIdx.x & (L - 1), at_once = kThreads / L, mine = threadIdx.x / L;
  constexpr bool KEEP = ROW_THREADS == 64;  // weights in registers; rows of more elements leave no room for them
  float w[KEEP ? P : 1][V], dw[P][V];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (lane + i * L) * V;
    if constexpr (KEEP) load_params<V>(a.weight, a.weight_dtype, at, a.dim - at, w[i]);
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i][j] = 0.0f;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * at_once; row0 < a.rows; row0 += (int64_t)gridDim.x * at_once) {
    const bool there = row0 + mine < a.rows;
    const int64_t row = there ? row0 + mine : a.rows - 1;
    const float rstd = a.rstd[row];
    float s[P][V], d[P][V], dot = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      load_floats<S, V>((const S *)a.s + row * a.ss + at, a.dim - at, s[i]);
      load_floats<E, V>((const E *)a.dout + row * a.dos + at, a.dim - at, d[i]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      if constexpr (!KEEP) load_params<V>(a.weight, a.weight_dtype, at, a.dim - at, w[0]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s[i][j] *= rstd;
        if (there) dw[i][j] += d[i][j] * s[i][j];
        d[i][j] *= w[KEEP ? i : 0][j];
        if (at + j < a.dim) dot += d[i][j] * s[i][j];
      }
    }
    dot = row_sum<ROW_THREADS>(dot, L, lds) / (float)a.dim;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      float g[V];
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = rstd * (d[i][j] - s[i][j] * dot);
      if (a.ds) {
        float o[V];
        load_floats<S, V>((const S *)a.ds + row * a.dss + at, a.dim - at, o);
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] += o[j];
      }
      if (there && a.dx) store_floats<E, V>((E *)a.dx + row * a.dxs + at, a.dim - at, g);
      if (there && a.dres) store_floats<S, V>((S *)a.dres + row * a.drs + at, a.dim - at, g);
    }
  }
  if (!a.parts) return;
  if constexpr (ROW_THREADS > 64) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (lane + i * L) * V;
      store_floats<float, V>(a.parts + (int64_t)blockIdx.x * a.dim + at, a.dim - at, dw[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sums[(mine * P + i) * L * V + lane * V + j] = dw[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += kThreads) {
      float v = 0.0f;
      for (int m = 0; m < at_once; ++m) v += sums[m * P * L * V + c];
      a.parts[(int64_t)blockIdx.x * a.dim + c] = v;
    }
  }
}

// The same of rows of so many elements that no lane keeps its part: the inputs are read twice (the second time from the cache), and the sums of dw
// lie in `parts` from the first row on, where each lane adds to its own columns.
constexpr int kWideThreads = 1024;
template <class E, class S>
__global__ __launch_bounds__(kWideThreads) void norm_grad_wide_kernel(NormGrad a) {
  constexpr int V = kPack<E>, L = kWideThreads;
  __shared__ float lds[L / 64];
  const int packs = (a.dim + V - 1) / V;
  float *part = a.parts ? a.parts + (int64_t)blockIdx.x * a.dim : nullptr;
  if (part && blockIdx.x >= a.rows)
    for (int at = threadIdx.x; at < a.dim; at += L) part[at] = 0.0f;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row];
    float dot = 0.0f, s[V], d[V], w[V];
    auto take = [&](int at) {
      load_floats<S, V>((const S *)a.s + row * a.ss + at, a.dim - at, s);
      load_floats<E, V>((const E *)a.dout + row * a.dos + at, a.dim - at, d);
      load_params<V>(a.weight, a.weight_dtype, at, a.dim - at, w);
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] *= rstd;
    };
    for (int p = threadIdx.x; p < packs; p += L) {
      const int at = p * V;
      take(at);
      float t[V];
      if (part && row >= gridDim.x) load_floats<float, V>(part + at, a.dim - at, t);
      else
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        t[j] += d[j] * s[j];
        if (at + j < a.dim) dot += d[j] * w[j] * s[j];
      }
      if (part) store_floats<float, V>(part + at, a.dim - at, t);
    }
    dot = row_sum<L>(dot, L, lds) / (float)a.dim;
    for (int p = threadIdx.x; p < packs; p += L) {
      const int at = p * V;
      take(at);
      float g[V];
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = rstd * (d[j] * w[j] - s[j] * dot);
      if (a.ds) {
        float o[V];
        load_floats<S, V>((const S *)a.ds + row * a.dss + at, a.dim - at, o);
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] += o[j];
      }
      if (a.dx) store_floats<E, V>((E *)a.dx + row * a.dxs + at, a.dim - at, g);
      if (a.dres) store_floats<S, V>((S *)a.dres + row * a.drs + at, a.dim - at, g);
    }
  }
}

// How a row lies on lanes: on a part of a wavefront or a whole one (threads 64, up to two packs a lane), on 256 or on 1024 lanes of up to 32 elements
constexpr int kElements = 32, kMostDim = 1024 * kElements;
template <class E> constexpr int kHalf = kElements / kPack<E> / 2;
struct Lay {
  int threads, lanes, packs;
};
Lay lay_of(int dim, int V) {
  const int64_t n = divide_up(dim, V);
  if (dim > 256 * kElements) return {1024, 1024, kElements / V};
  if (n > 128) return {256, 256, dim > 128 * kElements ? kElements / V : kElements / V / 2};  // up to 16 elements, or up to 32
  int lanes = 1;
  while (lanes < n && lanes < 64) lanes *= 2;
  return {64, lanes, n > 64 ? 2 : 1};
}

template <class E, class R, bool BITS8>
void launch_norm(NormArgs a, hipStream_t st) {
  const Lay l = lay_of(a.dim, kPack<E>);
  a.lanes = l.lanes;
  const int threads = l.threads > 64 ? l.threads : kThreads, at_once = threads / l.lanes;
  const int64_t groups = divide_up(a.rows, at_once);
  for (int64_t done = 0; done < groups; done += most_groups(threads)) {  // one launch, unless there are 2^32 lanes
    const dim3 grid((unsigned)std::min(groups - done, most_groups(threads)));
    a.row0 = done * at_once;
    if (l.threads == 64 && l.packs == 1) norm_kernel<E, R, BITS8, 64, 1><<<grid, threads, 0, st>>>(a);
    else if (l.threads == 64) norm_kernel<E, R, BITS8, 64, 2><<<grid, threads, 0, st>>>(a);
    else if (l.threads == 256 && l.packs == kHalf<E>) norm_kernel<E, R, BITS8, 256, kHalf<E>><<<grid, threads, 0, st>>>(a);
    else if (l.threads == 256) norm_kernel<E, R, BITS8, 256, 2 * kHalf<E>><<<grid, threads, 0, st>>>(a);
    else norm_kernel<E, R, BITS8, 1024, 2 * kHalf<E>><<<grid, threads, 0, st>>>(a);
  }
}

int64_t grad_groups(int64_t rows, int dim, Lay l) {
  const int at_once = l.threads > 64 ? 1 : kThreads / l.lanes;
  return std::max<int64_t>(1, std::min({divide_up(rows, at_once), kMostParts, std::max<int64_t>(256, kPartFloats / dim)}));
}

template <class E, class S>
void launch_grad(NormGrad a, float *dweight, hipStream_t st) {
  const Lay l = lay_of(a.dim, kPack<E>);
  a.lanes = l.lanes;
  const int64_t groups = grad_groups(a.rows, a.dim, l);
  const dim3 grid((unsigned)groups);
  const size_t lds = (size_t)kThreads * kPack<E> * l.packs * sizeof(float);
  if (l.threads == 64 && l.packs == 1) norm_grad_kernel<E, S, 64, 1><<<grid, kThreads, lds, st>>>(a);
  else if (l.threads == 64) norm_grad_kernel<E, S, 64, 2><<<grid, kThreads, lds, st>>>(a);
  else if (l.threads == 256 && l.packs == kHalf<E>) norm_grad_kernel<E, S, 256, kHalf<E>><<<grid, kThreads, 0, st>>>(a);
  else if (l.threads == 256) norm_grad_kernel<E, S, 256, 2 * kHalf<E>><<<grid, kThreads, 0, st>>>(a);
  else norm_grad_wide_kernel<E, S><<<grid, kWideThreads, 0, st>>>(a);
  if (dweight) sum_parts(a.parts, groups, a.dim, a.dim, a.dim, dweight, nullptr, nullptr, st);
}

}  // namespace

struct tbe_norm_t : DenseBase {
  int dim, dtype, residual_dtype;  // residual_dtype -1: no residual
  float eps;
  int64_t max_rows;
  float *parts = nullptr;
};

namespace {

template <bool BITS8>
void launch_typed(tbe_norm_handle s, const NormArgs &a, bool residual, hipStream_t st) {
  const bool wide = s->residual_dtype == TBE_FP32;
  if (s->dtype == TBE_FP32) return residual ? launch_norm<float, float, BITS8>(a, st) : launch_norm<float, void, BITS8>(a, st);
  if (s->dtype == TBE_FP16)
    return !residual ? launch_norm<_Float16, void, BITS8>(a, st) : wide ? launch_norm<_Float16, float, BITS8>(a, st) : launch_norm<_Float16, _Float16, BITS8>(a, st);
  return !residual ? launch_norm<__bf16, void, BITS8>(a, st) : wide ? launch_norm<__bf16, float, BITS8>(a, st) : launch_norm<__bf16, __bf16, BITS8>(a, st);
}

int check_rows(tbe_norm_handle s, int64_t rows) {
  if (int rc = check_handle(s)) return rc;
  if (rows < 0) return report(TBE_EINVAL, "negative number of rows");
  if (rows > s->max_rows) return report(TBE_ELIMIT, "more rows than the handle was created for");
  return TBE_OK;
}

int forward(tbe_norm_handle s, const tbe_norm_batch *b, void *out, int64_t os, float *rstd, float *scales, int32_t group, bool bits8, void *stream) {
  if (!b) return report(TBE_EINVAL, "null batch");
  if (int rc = check_rows(s, b->rows)) return rc;
  const bool residual = b->d_residual != nullptr;
  if (residual && s->residual_dtype < 0) return report(TBE_EINVAL, "the handle was created without a residual");
  if (!known_dtype(b->weight_dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (b->rows == 0) return TBE_OK;
  if (!b->d_x || !b->d_weight || !out || (residual && !b->d_summed) || (bits8 && !scales)) return report(TBE_EINVAL, "null rows, weights or results");
  if (b->x_stride < s->dim || os < s->dim || (residual && (b->residual_stride < s->dim || b->summed_stride < s->dim)))
    return report(TBE_EINVAL, "a stride below dim");
  if (residual && ((b->d_summed == b->d_residual && b->summed_stride != b->residual_stride) ||
                   (b->d_summed == b->d_x && (b->summed_stride != b->x_stride || s->dtype != s->residual_dtype))))
    return report(TBE_EINVAL, "a sum in place of an input has its type and strides");
  const int bytes = elem_bytes(s->dtype), res_bytes = residual ? elem_bytes(s->residual_dtype) : 0;
  const int64_t groups = group && group < s->dim ? divide_up(s->dim, group) : 1;
  const Span x = span(b->d_x, s->dim, b->x_stride, b->rows, bytes), res = span(residual ? b->d_residual : nullptr, s->dim, b->residual_stride, b->rows, res_bytes);
  const Span sum = span(residual ? b->d_summed : nullptr, s->dim, b->summed_stride, b->rows, res_bytes), weight = span(b->d_weight, (int64_t)s->dim * elem_bytes(b->weight_dtype));
  if (int rc = check_apart({span(out, s->dim, os, b->rows, bits8 ? 1 : bytes), span(rstd, b->rows * 4), span(scales, b->rows * groups * 4)}, {x, res, sum, weight})) return rc;
  if (int rc = check_apart({sum}, {same_span(sum, x) ? Span{} : x, same_span(sum, res) ? Span{} : res, weight})) return rc;
  NormArgs a{};
  a.x = b->d_x, a.residual = b->d_residual, a.weight = b->d_weight;
  a.xs = b->x_stride, a.rs = b->residual_stride, a.rows = b->rows;
  a.dim = s->dim, a.weight_dtype = b->weight_dtype, a.eps = s->eps;
  a.out = out, a.summed = b->d_summed, a.os = os, a.ss = b->summed_stride;
  a.rstd = rstd, a.scales = scales;
  a.group = group && group < s->dim ? group : s->dim;
  a.groups = (int)divide_up(s->dim, a.group);
  if (bits8) launch_typed<true>(s, a, residual, (hipStream_t)stream);
  else launch_typed<false>(s, a, residual, (hipStream_t)stream);
  return check_launch();
}

}  // namespace

extern "C" {

int tbe_norm_create(tbe_norm_handle *out, int32_t dim, int32_t dtype, int32_t residual_dtype, double eps, int64_t max_rows) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (dim < 1 || dim > kMostDim) return report(TBE_EINVAL, "dim outside 1 .. 32768");
  if (!known_dtype(dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (residual_dtype != -1 && residual_dtype != dtype && residual_dtype != TBE_FP32) return report(TBE_EINVAL, "the residual is of the rows' type or fp32");
  if (!(eps >= 0.0) || eps > 1e30) return report(TBE_EINVAL, "eps is negative or no number");
  if (max_rows < 0) return report(TBE_EINVAL, "negative number of rows");
  if (max_rows > (1ll << 40) / dim) return report(TBE_ELIMIT, "more than 2^40 elements");
  tbe_norm_t *s = new (std::nothrow) tbe_norm_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->dim = dim, s->dtype = dtype, s->residual_dtype = residual_dtype, s->eps = (float)eps, s->max_rows = max_rows;
  const Lay l = lay_of(dim, 16 / elem_bytes(dtype));
  const int64_t groups = grad_groups(max_rows, dim, l);
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&s->parts, (size_t)groups * dim * sizeof(float));
  if (e != hipSuccess) {
    delete s;
    return report_hip(e);
  }
  *out = s;
  return TBE_OK;
}

int tbe_norm_destroy(tbe_norm_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->parts);
  delete s;
  return TBE_OK;
}

int tbe_norm_forward(tbe_norm_handle s, const tbe_norm_batch *batch, void *d_out, int64_t out_stride, float *d_rstd, void *stream) {
  return forward(s, batch, d_out, out_stride, d_rstd, nullptr, 0, false, stream);
}

int tbe_norm_quantise(tbe_norm_handle s, const tbe_norm_batch *batch, int32_t group, void *d_codes, int64_t codes_stride, float *d_scales, void *stream) {
  if (group != 0 && (group < 16 || group > 256 || (group & (group - 1)))) return report(TBE_EINVAL, "a group is 0 (a row) or a power of two from 16 to 256");
  return forward(s, batch, d_codes, codes_stride, nullptr, d_scales, group, true, stream);
}

int tbe_norm_backward(tbe_norm_handle s, const tbe_norm_grad *g, void *stream) {
  if (!g) return report(TBE_EINVAL, "null gradients");
  if (int rc = check_rows(s, g->rows)) return rc;
  if (!known_dtype(g->weight_dtype)) return report(TBE_EINVAL, "unknown dtype");
  const bool residual = s->residual_dtype >= 0 && g->residual;
  if (g->residual && s->residual_dtype < 0) return report(TBE_EINVAL, "the handle was created without a residual");
  if (g->d_dresidual && !residual) return report(TBE_EINVAL, "a gradient of a residual that there is not");
  if (g->rows == 0 && !g->d_dweight) return TBE_OK;
  if (!g->d_weight || (g->rows > 0 && (!g->d_summed || !g->d_rstd || !g->d_dout))) return report(TBE_EINVAL, "null rows, weights or gradients");
  if (g->rows > 0 && (g->summed_stride < s->dim || g->dout_stride < s->dim || (g->d_dsummed && g->dsummed_stride < s->dim) ||
                      (g->d_dx && g->dx_stride < s->dim) || (g->d_dresidual && g->dresidual_stride < s->dim)))
    return report(TBE_EINVAL, "a stride below dim");
  const int bytes = elem_bytes(s->dtype), sum_bytes = residual ? elem_bytes(s->residual_dtype) : bytes;
  if (int rc = check_apart({span(g->d_dx, s->dim, g->dx_stride, g->rows, bytes), span(g->d_dresidual, s->dim, g->dresidual_stride, g->rows, sum_bytes), span(g->d_dweight, (int64_t)s->dim * 4)},
                           {span(g->d_summed, s->dim, g->summed_stride, g->rows, sum_bytes), span(g->d_dout, s->dim, g->dout_stride, g->rows, bytes),
                            span(g->d_dsummed, s->dim, g->dsummed_stride, g->rows, sum_bytes), span(g->d_weight, (int64_t)s->dim * elem_bytes(g->weight_dtype)), span(g->d_rstd, g->rows * 4)}))
    return rc;
  NormGrad a{};
  a.s = g->d_summed, a.dout = g->d_dout, a.ds = g->d_dsummed, a.weight = g->d_weight;
  a.ss = g->summed_stride, a.dos = g->dout_stride, a.dss = g->dsummed_stride, a.rows = g->rows;
  a.dim = s->dim, a.weight_dtype = g->weight_dtype, a.rstd = g->d_rstd;
  a.dx = g->d_dx, a.dres = g->d_dresidual, a.dxs = g->dx_stride, a.drs = g->dresidual_stride;
  a.parts = g->d_dweight ? s->parts : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const bool wide = residual && s->residual_dtype == TBE_FP32;
  if (s->dtype == TBE_FP32) launch_grad<float, float>(a, g->d_dweight, st);
  else if (s->dtype == TBE_FP16) wide ? launch_grad<_Float16, float>(a, g->d_dweight, st) : launch_grad<_Float16, _Float16>(a, g->d_dweight, st);
  else wide ? launch_grad<__bf16, float>(a, g->d_dweight, st) : launch_grad<__bf16, __bf16>(a, g->d_dweight, st);
  return check_launch();
}

}  // extern "C"
