// Learned bias by the bucket of a distance: values (alone or added to scores) and the gradient of the table.
// Contract: include/tbe.h.
//
// The bucket of a (query, key) pair is the same for all heads, so a lane finds those of V neighbouring keys (16 bytes of scores) once
// and goes through the heads with them.  A bucket is found in two looks at LDS: the distance's exponent and 6 bits of its
// mantissa name a cell, the cell the number of thresholds that everything in it reaches, and one comparison decides about the next
// one.  (Where a cell holds more thresholds than one, as many comparisons as it takes.)
#include <cmath>
#include <new>

#include "tbe_dense.h"
#include "tbe_internal.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxThresholds = 127;
constexpr int kCells = 4096;                 // 64 an octave up to 2^63, and one for distance zero
constexpr int kTableFloats = 8192;           // of the table in LDS: heads of a workgroup times buckets
constexpr int kSums = 4096;                  // numbers of a wavefront's sums in LDS (gradient)
constexpr int kMaxParts = 1024;              // workgroups whose sums of a head are added up

struct Buckets {  // in device memory
  int64_t threshold[kMaxThresholds + 1];  // behind the last one: INT64_MAX
  uint8_t reached[kCells];                // thresholds that all distances of a cell reach
};

struct Shape {
  tbe_bias_shape s;
  int heads, thresholds, buckets;  // buckets of the whole table
  bool both, dense;                // dense: a cell holds several thresholds
  const Buckets *map;              // device
  uint32_t packs;                  // of a row
  unsigned long long packs_magic;
};

struct Finder {  // in LDS
  int64_t threshold[kMaxThresholds + 1];
  uint8_t reached[kCells];
};

__device__ inline void load_finder(const Shape &p, Finder &f) {
  static_assert(sizeof(Finder) == sizeof(Buckets) && sizeof(Finder) % 16 == 0, "copied as it is");
  for (int k = threadIdx.x; k < (int)(sizeof(Finder) / 16); k += kThreads) ((uint4 *)&f)[k] = ((const uint4 *)p.map)[k];
}

// cell of a distance: monotone, and exact at the cells' borders below 2^22 (above, a distance just below a border may count as on it,
// which the cells' numbers allow for)
__host__ __device__ inline int cell_of(uint64_t a) {
  const float f = (float)(uint32_t)(a >> 32) * 4294967296.0f + (float)(uint32_t)a;
  uint32_t bits;
  __builtin_memcpy(&bits, &f, 4);
  const int c = (int)(bits >> 17) - (127 * 64 - 1);
  return c > 0 ? c : 0;
}

// bucket of a key `ahead` positions after the query
__device__ inline int bucket_of(const Shape &p, const Finder &f, int64_t ahead) {
  const int64_t d = min(ahead < 0 ? -ahead : (p.both ? ahead : 0), INT64_MAX - 1);  // below the number behind the last threshold
  int b = f.reached[cell_of((uint64_t)d)];
  b += d >= f.threshold[b];
  if (p.dense)
    while (d >= f.threshold[b]) b++;
  return b + (p.both && ahead > 0 ? p.thresholds + 1 : 0);
}

__device__ inline float table_value(const void *table, int dtype, int64_t i) {
  if (dtype == TBE_FP32) return ((const float *)table)[i];
  if (dtype == TBE_FP16) return (float)((const _Float16 *)table)[i];
  return (float)((const __bf16 *)table)[i];
}

// V keys of a query: their buckets, and which of them are masked
template <int V>
struct Keys {
  int64_t i, j;
  int n;               // keys that there are
  int bucket[V];
  uint32_t masked;     // bits
};

template <int V>
__device__ inline void find_keys(const Shape &p, const Finder &f, int64_t b, int64_t item, Keys<V> &k) {
  k.i = (int64_t)div_by((uint32_t)item, p.packs_magic);
  k.j = (item - k.i * p.packs) * V;
  k.n = (int)min((int64_t)V, p.s.keys - k.j);
  const int64_t q = p.s.d_query_pos ? p.s.d_query_pos[b * p.s.query_pos_stride + k.i] : p.s.query_offset + k.i;
  const int64_t len = p.s.d_key_lengths ? p.s.d_key_lengths[b] : p.s.keys;
  int64_t ahead[V];
  if (p.s.d_key_pos) {
    const int64_t *kp = p.s.d_key_pos + b * p.s.key_pos_stride + k.j;
#pragma unroll
    for (int v = 0; v < V; v++) ahead[v] = kp[min(v, k.n - 1)] - q;
  } else {
#pragma unroll
    for (int v = 0; v < V; v++) ahead[v] = k.j + v - q;
  }
  k.masked = 0;
#pragma unroll
  for (int v = 0; v < V; v++) {
    k.bucket[v] = bucket_of(p, f, ahead[v]);
    const bool later = p.s.causal && ahead[v] > 0, beyond = k.j + v >= len;
    k.masked |= (later | beyond) ? 1u << v : 0u;
  }
}

template <class E, int V>
__device__ inline Pack<E, V> read_pack(const E *p) {  // at any address that an element may have
  Pack<E, V> r;
  __builtin_memcpy(&r, p, sizeof r);
  return r;
}
template <class E, int V>
__device__ inline void write_pack(E *p, const Pack<E, V> &r) {
  __builtin_memcpy(p, &r, sizeof r);
}

// A workgroup has a group of heads (blockIdx.y), whose part of the table it keeps in LDS, and of all samples' packs of keys every
// gridDim.x-th 256.
template <int DT, bool SCORES>
__global__ __launch_bounds__(kThreads) void bias_forward_kernel(Shape p, int group, const void *table, int table_dtype, const typename Elem<DT>::type *scores,
                                                                tbe_bias_strides ss, float scale, float mask, typename Elem<DT>::type *out,
                                                                tbe_bias_strides os) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E);
  __shared__ __align__(16) Finder find;
  extern __shared__ float value[];  // [group][buckets]
  const int h0 = blockIdx.y * group, heads = min(group, p.heads - h0);
  load_finder(p, find);
  for (int k = threadIdx.x; k < heads * p.buckets; k += kThreads)
    value[k] = table_value(table, table_dtype, (int64_t)(k % p.buckets) * p.heads + h0 + k / p.buckets);
  __syncthreads();
  const int64_t items = p.s.queries * p.packs, blocks = (items + kThreads - 1) / kThreads;
  for (int64_t w = blockIdx.x; w < blocks * p.s.batch; w += gridDim.x) {
    const int64_t b = w / blocks, item = (w - b * blocks) * kThreads + threadIdx.x;
    if (item >= items) continue;
    Keys<V> k;
    find_keys<V>(p, find, b, item, k);
    const E *in = SCORES ? scores + b * ss.sample + h0 * ss.head + k.i * ss.query + k.j : nullptr;
    E *to = out + b * os.sample + h0 * os.head + k.i * os.query + k.j;
    const bool whole = k.n == V, blank = k.masked == (1u << V) - 1;
#pragma unroll 4
    for (int h = 0; h < heads; h++) {
      Pack<E, V> x = {}, y;
      if (SCORES && !blank) {
        if (whole) x = read_pack<E, V>(in + h * ss.head);
        else
#pragma unroll
          for (int v = 0; v < V; v++) x.e[v] = in[h * ss.head + min(v, k.n - 1)];
      }
#pragma unroll
      for (int v = 0; v < V; v++) {
        float r = value[h * p.buckets + k.bucket[v]];
        if (SCORES) r += (float)x.e[v] * scale;
        y.e[v] = (E)(k.masked >> v & 1 ? mask : r);
      }
      if (whole) write_pack<E, V>(to + h * os.head, y);
      else
#pragma unroll
        for (int v = 0; v < V; v++)
          if (v < k.n) to[h * os.head + v] = y.e[v];
    }
  }
}

// Gradient of the table.  A wavefront has sums of its own in LDS, [heads of the group][buckets][slots], a lane adds to slot lane % slots:
// one wavefront's additions come in one order, so the sums do not depend on how the wavefronts run.
template <int DT, bool SCORES>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(Shape p, int group, int slots, const typename Elem<DT>::type *dout, tbe_bias_strides ds,
                                                             float *part, float scale, typename Elem<DT>::type *dscores, tbe_bias_strides es) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E);
  __shared__ __align__(16) Finder find;
  extern __shared__ float sums[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h0 = blockIdx.y * group, heads = min(group, p.heads - h0);
  const int head_floats = p.buckets * slots, own = group * head_floats;
  float *sum = sums + wave * own + (lane & (slots - 1));
  load_finder(p, find);
  for (int k = threadIdx.x; k < kWaves * own; k += kThreads) sums[k] = 0.0f;
  __syncthreads();
  const int64_t items = p.s.queries * p.packs, blocks = (items + kThreads - 1) / kThreads;
  for (int64_t w = blockIdx.x; w < blocks * p.s.batch; w += gridDim.x) {
    const int64_t b = w / blocks, item = (w - b * blocks) * kThreads + threadIdx.x;
    if (item >= items) continue;
    Keys<V> k;
    find_keys<V>(p, find, b, item, k);
    const E *in = dout + b * ds.sample + h0 * ds.head + k.i * ds.query + k.j;
    const bool whole = k.n == V, blank = k.masked == (1u << V) - 1;
#pragma unroll 4
    for (int h = 0; h < heads; h++) {
      Pack<E, V> x = {};
      if (!blank) {
        if (whole) x = read_pack<E, V>(in + h * ds.head);
        else
#pragma unroll
          for (int v = 0; v < V; v++) x.e[v] = in[h * ds.head + min(v, k.n - 1)];
      }
#pragma unroll
      for (int v = 0; v < V; v++) {
        const bool on = !(k.masked >> v & 1) && v < k.n;
        if (on) unsafeAtomicAdd(sum + h * head_floats + k.bucket[v] * slots, (float)x.e[v]);
        if (SCORES) x.e[v] = (E)(on ? (float)x.e[v] * scale : 0.0f);
      }
      if (SCORES) {
        E *to = dscores + b * es.sample + (h0 + h) * es.head + k.i * es.query + k.j;
        if (whole) write_pack<E, V>(to, x);
        else
#pragma unroll
          for (int v = 0; v < V; v++)
            if (v < k.n) to[v] = x.e[v];
      }
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < heads * p.buckets; k += kThreads) {
    float v = 0.0f;
    for (int w = 0; w < kWaves; w++)
      for (int s = 0; s < slots; s++) v += sums[w * own + k * slots + ((s + lane) & (slots - 1))];
    part[((int64_t)blockIdx.x * p.heads + h0) * p.buckets + k] = v;
  }
}

// a wavefront for each number of the table's gradient
__global__ __launch_bounds__(kThreads) void bias_join_kernel(const float *part, int parts, int heads, int buckets, float *dtable) {
  const int id = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63, h = id / buckets, c = id % buckets;
  if (h >= heads) return;
  float v = 0.0f;
#pragma unroll 4
  for (int k = lane; k < parts; k += 64) v += part[((int64_t)k * heads + h) * buckets + c];
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  if (lane == 0) dtable[(int64_t)c * heads + h] = v;
}

}  // namespace

struct tbe_bias_t : DenseBase {
  int heads = 0, thresholds = 0, buckets = 0;
  bool both = false, dense = false;
  Buckets *map = nullptr;  // device
  float *part = nullptr;   // device [kMaxParts, heads, buckets]
};

namespace {

int check_shape(tbe_bias_t *s, const tbe_bias_shape *p, Shape *out) noexcept {
  if (int rc = check_handle(s)) return rc;
  if (!p) return report(TBE_EINVAL, "null shape");
  if (p->batch < 0 || p->queries < 0 || p->keys < 0) return report(TBE_EINVAL, "a negative size");
  if (!known_dtype(p->dtype)) return report(TBE_EINVAL, "unknown dtype");
  const int V = 16 / elem_bytes(p->dtype);
  if (p->batch > INT32_MAX || p->queries > INT32_MAX || p->keys > INT32_MAX || (double)p->queries * (double)p->keys > 0x1p31 ||
      (double)p->batch * s->heads * (double)p->queries * (double)p->keys > 0x1p40)
    return report(TBE_ELIMIT, "more than 2^31 scores of a head, or 2^40 scores");
  if ((p->d_query_pos && p->query_pos_stride != 0 && p->query_pos_stride < p->queries) ||
      (p->d_key_pos && p->key_pos_stride != 0 && p->key_pos_stride < p->keys))
    return report(TBE_EINVAL, "a stride of positions that is neither 0 nor as long as a sample's");
  const uint32_t packs = (uint32_t)((p->keys + V - 1) / V);
  *out = {*p, s->heads, s->thresholds, s->buckets, s->both, s->dense, s->map, packs, div_magic(packs)};
  return TBE_OK;
}

int64_t blocks_of(const Shape &p) { return (p.s.queries * p.packs + kThreads - 1) / kThreads * p.s.batch; }

}  // namespace

extern "C" {

int tbe_bias_destroy(tbe_bias_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->map);
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
    if (h_thresholds[k] < (k ? h_thresholds[k - 1] + 1 : 1) || h_thresholds[k] == INT64_MAX)
      return report(TBE_EINVAL, "thresholds ascend from 1 or more");
  tbe_bias_t *s = new (std::nothrow) tbe_bias_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->heads = heads;
  s->thresholds = num_thresholds;
  s->both = bidirectional != 0;
  s->buckets = (num_thresholds + 1) * (s->both ? 2 : 1);
  Buckets map;
  for (int k = 0; k <= kMaxThresholds; k++) map.threshold[k] = k < num_thresholds ? h_thresholds[k] : INT64_MAX;
  for (int c = 0; c < kCells; c++) {  // distances lo .. hi can lie in the cell; the next cell's border is hi + 1
    int64_t lo = 0, hi = 0;
    if (c > 0) {
      const double from = std::ldexp(1.0 + ((c - 1) % 64) / 64.0, (c - 1) / 64), to = std::ldexp(1.0 + (c - 1) % 64 / 64.0 + 1.0 / 64.0, (c - 1) / 64);
      const double below = from >= 4194304.0 ? from * (1.0 - 0x1p-22) : from;
      lo = below >= 0x1p63 ? INT64_MAX - 1 : (int64_t)std::ceil(below);
      hi = to >= 0x1p63 ? INT64_MAX - 1 : (int64_t)std::ceil(to) - 1;
    }
    int all = 0, some = 0;
    for (int k = 0; k < num_thresholds; k++) {
      all += h_thresholds[k] <= lo;
      some += h_thresholds[k] <= hi;
    }
    map.reached[c] = (uint8_t)all;
    s->dense |= some - all > 1;
  }
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&s->map, sizeof(Buckets));
  if (e == hipSuccess) e = hipMalloc((void **)&s->part, (size_t)kMaxParts * heads * s->buckets * sizeof(float));
  if (e == hipSuccess) e = hipMemcpy(s->map, &map, sizeof map, hipMemcpyHostToDevice);
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
  if (p.s.batch * p.s.queries * p.s.keys == 0) return TBE_OK;
  if (!d_table || !d_out || !out_strides || (d_scores && !scores_strides)) return report(TBE_EINVAL, "null table, output or strides");
  const tbe_bias_strides ss = d_scores ? *scores_strides : tbe_bias_strides{0, 0, 0};
  const int group = p.heads < kTableFloats / p.buckets ? p.heads : kTableFloats / p.buckets, groups = (p.heads + group - 1) / group;
  const int64_t blocks = blocks_of(p);
  const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), (unsigned)groups);
  const size_t lds = (size_t)group * p.buckets * sizeof(float);
#define LAUNCH(DT, SCORES)                                                                                                              \
  bias_forward_kernel<DT, SCORES><<<grid, kThreads, lds, (hipStream_t)stream>>>(p, group, d_table, table_dtype, (const Elem<DT>::type *)d_scores, ss, \
                                                                                scale, mask_value, (Elem<DT>::type *)d_out, *out_strides)
#define LAUNCH2(DT) (d_scores ? LAUNCH(DT, true) : LAUNCH(DT, false))
  if (p.s.dtype == TBE_FP32) LAUNCH2(TBE_FP32);
  else if (p.s.dtype == TBE_FP16) LAUNCH2(TBE_FP16);
  else LAUNCH2(TBE_BF16);
#undef LAUNCH2
#undef LAUNCH
  return check_launch();
}

int tbe_bias_backward(tbe_bias_handle s, const tbe_bias_shape *shape, const void *d_dout, const tbe_bias_strides *dout_strides, float *d_dtable,
                      float scale, void *d_dscores, const tbe_bias_strides *dscores_strides, void *stream) {
  Shape p;
  if (int rc = check_shape(s, shape, &p)) return rc;
  const bool any = p.s.batch * p.s.queries * p.s.keys != 0;
  if (any && (!d_dout || !dout_strides || (d_dscores && !dscores_strides))) return report(TBE_EINVAL, "null gradient or strides");
  const tbe_bias_strides es = d_dscores ? *dscores_strides : tbe_bias_strides{0, 0, 0};
  int parts = 0;
  if (any) {
    int group = 1, slots = 64;
    while (slots > 1 && p.buckets * slots > kSums) slots /= 2;
    while (group < p.heads && group < 16 && (2 * group * p.buckets * slots <= kSums || (slots > 16 && 2 * group * p.buckets * 16 <= kSums))) {
      group *= 2;
      while (slots > 16 && group * p.buckets * slots > kSums) slots /= 2;
    }
    const int64_t blocks = blocks_of(p);
    parts = (int)(blocks < kMaxParts ? blocks : kMaxParts);
    const dim3 grid((unsigned)parts, (unsigned)((p.heads + group - 1) / group));
    const size_t lds = (size_t)kWaves * group * p.buckets * slots * sizeof(float);
#define LAUNCH(DT, SCORES)                                                                                                                 \
  bias_grad_kernel<DT, SCORES><<<grid, kThreads, lds, (hipStream_t)stream>>>(p, group, slots, (const Elem<DT>::type *)d_dout, *dout_strides, s->part, \
                                                                             scale, (Elem<DT>::type *)d_dscores, es)
#define LAUNCH2(DT) (d_dscores ? LAUNCH(DT, true) : LAUNCH(DT, false))
    if (p.s.dtype == TBE_FP32) LAUNCH2(TBE_FP32);
    else if (p.s.dtype == TBE_FP16) LAUNCH2(TBE_FP16);
    else LAUNCH2(TBE_BF16);
#undef LAUNCH2
#undef LAUNCH
  }
  if (d_dtable)
    bias_join_kernel<<<dim3((unsigned)((p.heads * p.buckets + kWaves - 1) / kWaves)), kThreads, 0, (hipStream_t)stream>>>(s->part, parts, p.heads,
                                                                                                                        p.buckets, d_dtable);
  return check_launch();
}

}  // extern "C"
