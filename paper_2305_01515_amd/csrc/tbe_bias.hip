// Learned bias by the bucket of a distance: values (alone or added to scores) and the gradient of the table.
// Contract: include/tbe.h.
#include <cmath>
#include <new>

#include "tbe_dense.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxThresholds = 127;
constexpr int kMaxBuckets = 2 * (kMaxThresholds + 1);
constexpr int kMaxParts = 2048;  // workgroups whose sums the gradient's second kernel adds up, over all heads

struct Shape {
  tbe_bias_shape s;
  int heads, thresholds, buckets;  // buckets of the whole table
  bool both;
  const int64_t *threshold;        // device
};

__device__ inline int64_t query_at(const Shape &p, int64_t b, int64_t i) {
  return p.s.d_query_pos ? p.s.d_query_pos[b * p.s.query_pos_stride + i] : p.s.query_offset + i;
}
__device__ inline int64_t key_at(const Shape &p, int64_t b, int64_t j) { return p.s.d_key_pos ? p.s.d_key_pos[b * p.s.key_pos_stride + j] : j; }

// bucket of a key `ahead` positions after the query
__device__ inline int bucket_of(const Shape &p, const int64_t *thr, int64_t ahead) {
  const int64_t a = p.both ? (ahead < 0 ? -ahead : ahead) : (ahead < 0 ? -ahead : 0);
  int lo = 0, hi = p.thresholds;  // thresholds below lo are reached, those from hi on are not
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (thr[mid] <= a) lo = mid + 1;
    else hi = mid;
  }
  return lo + (p.both && ahead > 0 ? p.thresholds + 1 : 0);
}

__device__ inline float table_value(const void *table, int dtype, int64_t i) {
  if (dtype == TBE_FP32) return ((const float *)table)[i];
  if (dtype == TBE_FP16) return (float)((const _Float16 *)table)[i];
  return (float)((const __bf16 *)table)[i];
}

template <int DT>
__global__ __launch_bounds__(kThreads) void bias_forward_kernel(Shape p, const void *table, int table_dtype, const typename Elem<DT>::type *scores,
                                                                tbe_bias_strides ss, float scale, float mask, typename Elem<DT>::type *out,
                                                                tbe_bias_strides os) {
  using E = typename Elem<DT>::type;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t j = id % p.s.keys, i = id / p.s.keys % p.s.queries, h = id / p.s.keys / p.s.queries % p.heads, b = id / p.s.keys / p.s.queries / p.heads;
  if (b >= p.s.batch) return;
  const int64_t ahead = key_at(p, b, j) - query_at(p, b, i);
  float v = table_value(table, table_dtype, (int64_t)bucket_of(p, p.threshold, ahead) * p.heads + h);
  if (scores) v += (float)scores[b * ss.sample + h * ss.head + i * ss.query + j] * scale;
  const int64_t keys = p.s.d_key_lengths ? p.s.d_key_lengths[b] : p.s.keys;
  const bool later = p.s.causal && ahead > 0, beyond = j >= keys;
  v = (later | beyond) ? mask : v;  // a select: as a branch this was compiled to one that never took the mask
  out[b * os.sample + h * os.head + i * os.query + j] = (E)v;
}

// A workgroup takes every gridDim.x-th row of scores of head blockIdx.y; every lane has sums of its own.
template <int DT>
__global__ __launch_bounds__(64) void bias_grad_kernel(Shape p, const typename Elem<DT>::type *dout, tbe_bias_strides ds, float *part, float scale,
                                                       typename Elem<DT>::type *dscores, tbe_bias_strides es) {
  __shared__ float sum[kMaxBuckets * 64];
  const int lane = threadIdx.x, h = blockIdx.y;
  for (int c = 0; c < p.buckets; c++) sum[c * 64 + lane] = 0.0f;
  for (int64_t r = blockIdx.x; r < p.s.batch * p.s.queries; r += gridDim.x) {
    const int64_t b = r / p.s.queries, i = r % p.s.queries, q = query_at(p, b, i);
    const int64_t keys = p.s.d_key_lengths ? min(p.s.keys, p.s.d_key_lengths[b]) : p.s.keys;
    for (int64_t j = lane; j < p.s.keys; j += 64) {
      const int64_t ahead = key_at(p, b, j) - q;
      const bool masked = (p.s.causal && ahead > 0) || j >= keys;
      const float g = masked ? 0.0f : (float)dout[b * ds.sample + h * ds.head + i * ds.query + j];
      if (!masked) sum[bucket_of(p, p.threshold, ahead) * 64 + lane] += g;
      if (dscores) dscores[b * es.sample + h * es.head + i * es.query + j] = (typename Elem<DT>::type)(g * scale);
    }
  }
  for (int c = 0; c < p.buckets; c++) {
    float v = sum[c * 64 + lane];
    for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
    if (lane == 0) part[((int64_t)blockIdx.x * p.heads + h) * p.buckets + c] = v;
  }
}

__global__ __launch_bounds__(kThreads) void bias_join_kernel(const float *part, int parts, int heads, int buckets, float *dtable) {
  const int id = blockIdx.x * kThreads + threadIdx.x, h = id / buckets, c = id % buckets;
  if (h >= heads) return;
  float v = 0.0f;
  for (int k = 0; k < parts; k++) v += part[((int64_t)k * heads + h) * buckets + c];
  dtable[(int64_t)c * heads + h] = v;
}

}  // namespace

struct tbe_bias_t : DenseBase {
  int heads = 0, thresholds = 0, buckets = 0, parts = 0;
  bool both = false;
  int64_t *threshold = nullptr;  // device [thresholds]
  float *part = nullptr;         // device [parts, heads, buckets]
};

namespace {

int check_shape(tbe_bias_t *s, const tbe_bias_shape *p, Shape *out) noexcept {
  if (int rc = check_handle(s)) return rc;
  if (!p) return report(TBE_EINVAL, "null shape");
  if (p->batch < 0 || p->queries < 0 || p->keys < 0) return report(TBE_EINVAL, "a negative size");
  if (!known_dtype(p->dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (p->batch > INT32_MAX || p->queries > INT32_MAX || p->keys > INT32_MAX ||
      (double)p->batch * s->heads * (double)p->queries * (double)p->keys > 0x1p38)
    return report(TBE_ELIMIT, "more than 2^38 scores, or a size above 2^31");
  if ((p->d_query_pos && p->query_pos_stride != 0 && p->query_pos_stride < p->queries) ||
      (p->d_key_pos && p->key_pos_stride != 0 && p->key_pos_stride < p->keys))
    return report(TBE_EINVAL, "a stride of positions that is neither 0 nor as long as a sample's");
  *out = {*p, s->heads, s->thresholds, s->buckets, s->both, s->threshold};
  return TBE_OK;
}

}  // namespace

extern "C" {

int tbe_bias_destroy(tbe_bias_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->threshold);
  (void)hipFree(s->part);
  delete s;
  return TBE_OK;
}

int tbe_bias_create(tbe_bias_handle *out, int32_t heads, const int64_t *h_thresholds, int32_t num_thresholds, int32_t bidirectional) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (heads < 1 || heads > 4096) return report(TBE_EINVAL, "heads outside 1 .. 4096");
  if (num_thresholds < 0 || num_thresholds > kMaxThresholds) return report(TBE_EINVAL, "0 to 127 thresholds");
  if (num_thresholds && !h_thresholds) return report(TBE_EINVAL, "null thresholds");
  for (int k = 0; k < num_thresholds; k++)
    if (h_thresholds[k] < (k ? h_thresholds[k - 1] + 1 : 1)) return report(TBE_EINVAL, "thresholds ascend from 1 or more");
  tbe_bias_t *s = new (std::nothrow) tbe_bias_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->heads = heads;
  s->thresholds = num_thresholds;
  s->both = bidirectional != 0;
  s->buckets = (num_thresholds + 1) * (s->both ? 2 : 1);
  s->parts = kMaxParts / heads > 0 ? kMaxParts / heads : 1;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&s->threshold, (num_thresholds + 1) * sizeof(int64_t));
  if (e == hipSuccess) e = hipMalloc((void **)&s->part, (size_t)s->parts * heads * s->buckets * sizeof(float));
  if (e == hipSuccess && num_thresholds) e = hipMemcpy(s->threshold, h_thresholds, num_thresholds * sizeof(int64_t), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)tbe_bias_destroy(s);
    return report_hip(e);
  }
  *out = s;
  return TBE_OK;
}

int tbe_bias_forward(tbe_bias_handle s, const tbe_bias_shape *shape, const void *d_table, int32_t table_dtype, const void *d_scores,
                     const tbe_bias_strides *scores_strides, float scale, float mask_value, void *d_out, const tbe_bias_strides *out_strides,
                     void *stream) {
  Shape p;
  if (int rc = check_shape(s, shape, &p)) return rc;
  if (!known_dtype(table_dtype)) return report(TBE_EINVAL, "unknown dtype");
  const int64_t n = p.s.batch * p.heads * p.s.queries * p.s.keys;
  if (n == 0) return TBE_OK;
  if (!d_table || !d_out || !out_strides || (d_scores && !scores_strides)) return report(TBE_EINVAL, "null table, output or strides");
  const tbe_bias_strides ss = d_scores ? *scores_strides : tbe_bias_strides{0, 0, 0};
  const dim3 grid((unsigned)((n + kThreads - 1) / kThreads));
#define LAUNCH(DT)                                                                                                                       \
  bias_forward_kernel<DT><<<grid, kThreads, 0, (hipStream_t)stream>>>(p, d_table, table_dtype, (const Elem<DT>::type *)d_scores, ss, scale, mask_value, \
                                                            (Elem<DT>::type *)d_out, *out_strides)
  if (p.s.dtype == TBE_FP32) LAUNCH(TBE_FP32);
  else if (p.s.dtype == TBE_FP16) LAUNCH(TBE_FP16);
  else LAUNCH(TBE_BF16);
#undef LAUNCH
  return check_launch();
}

int tbe_bias_backward(tbe_bias_handle s, const tbe_bias_shape *shape, const void *d_dout, const tbe_bias_strides *dout_strides, float *d_dtable,
                      float scale, void *d_dscores, const tbe_bias_strides *dscores_strides, void *stream) {
  Shape p;
  if (int rc = check_shape(s, shape, &p)) return rc;
  const int64_t n = p.s.batch * p.heads * p.s.queries * p.s.keys;
  if (n > 0 && (!d_dout || !dout_strides || (d_dscores && !dscores_strides))) return report(TBE_EINVAL, "null gradient or strides");
  const tbe_bias_strides es = d_dscores ? *dscores_strides : tbe_bias_strides{0, 0, 0};
  const int64_t rows = p.s.batch * p.s.queries;
  const int parts = n == 0 ? 0 : (int)(rows < s->parts ? rows : s->parts);
  if (parts) {
    const dim3 grid((unsigned)parts, (unsigned)p.heads);
#define LAUNCH(DT) bias_grad_kernel<DT><<<grid, 64, 0, (hipStream_t)stream>>>(p, (const Elem<DT>::type *)d_dout, *dout_strides, s->part, scale, \
                                                           (Elem<DT>::type *)d_dscores, es)
    if (p.s.dtype == TBE_FP32) LAUNCH(TBE_FP32);
    else if (p.s.dtype == TBE_FP16) LAUNCH(TBE_FP16);
    else LAUNCH(TBE_BF16);
#undef LAUNCH
  }
  if (d_dtable) bias_join_kernel<<<dim3((unsigned)((p.heads * p.buckets + kThreads - 1) / kThreads)), kThreads, 0, (hipStream_t)stream>>>(s->part, parts, p.heads, p.buckets,
                                                                                                               d_dtable);
  return check_launch();
}

}  // extern "C"
