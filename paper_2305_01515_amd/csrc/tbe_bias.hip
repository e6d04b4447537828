// Learned bias by the bucket of a distance: values (alone or added to scores) and the gradient of the table.
// Contract: include/tbe.h.
//
// The bucket of a (query, key) pair is the same for all heads, so a lane finds those of V neighbouring keys (16 bytes of scores) once
// and goes through the heads with them.  A bucket is found in two looks at LDS: the distance's exponent and 6 bits of its
// mantissa name a cell, the cell the number of thresholds that everything in it reaches, and a comparison decides about the next
// one.  (As many comparisons as there are thresholds in the cell that has the most: one, unless thresholds beyond 128 are dense.)
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
constexpr int kSums = 2048;                  // numbers of a wavefront's sums of heads in LDS (gradient)
constexpr int kForward = 1024;               // workgroups of the forward
constexpr int kHeads = 4;                    // packs of scores on their way at once: as many heads
constexpr int kFill = 2048;                  // wavefronts that the gradient wants at least
constexpr size_t kLds = 160 << 10;            // of a CU
constexpr int kMaxParts = 1024;              // workgroups whose sums of a head are added up

struct Buckets {  // in device memory
  int64_t threshold[kMaxThresholds + 1];  // behind the last one: INT64_MAX
  uint8_t reached[kCells];                // thresholds that all distances of a cell reach
};

struct Shape {
  tbe_bias_shape s;
  int heads, thresholds, buckets;  // buckets of the whole table
  bool both;
  int steps;                       // thresholds that a cell holds at most (1 at least)
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
  for (int k = threadIdx.x; k < (int)(sizeof(Finder) / 16); k += blockDim.x) ((uint4 *)&f)[k] = ((const uint4 *)p.map)[k];
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

// the least number of a cell > 0
inline double border_of(int c) {
  const uint32_t bits = (uint32_t)(c + 127 * 64 - 1) << 17;
  float f;
  __builtin_memcpy(&f, &bits, 4);
  return f;
}

// bucket of a key `ahead` positions after the query
__device__ inline int bucket_of(const Shape &p, const Finder &f, int64_t ahead) {
  const int64_t back = -ahead, d = min(ahead > 0 ? (p.both ? ahead : 0) : back, INT64_MAX - 1);
  int b = f.reached[cell_of((uint64_t)d)];
  for (int s = 0; s < p.steps; s++) b += d >= f.threshold[b];
  return b + (p.both && ahead > 0 ? p.thresholds + 1 : 0);
}

__device__ inline float table_value(const void *table, int dtype, int64_t i) {
  if (dtype == TBE_FP32) return ((const float *)table)[i];
  if (dtype == TBE_FP16) return (float)((const _Float16 *)table)[i];
  return (float)((const __bf16 *)table)[i];
}

// V keys of a query: their buckets, and which of them are masked.  The last pack of a row is moved back to end where the row does; the
// keys that the pack before it has already are marked in `twice`.  (A row shorter than a pack has places without a key: n < V.)
template <int V>
struct Keys {
  int64_t i, j;
  int n;
  int bucket[V];
  uint32_t masked, twice;  // bits
};

template <int V>
__device__ inline void find_keys(const Shape &p, const Finder &f, int64_t b, uint32_t item, Keys<V> &k) {
  const uint32_t i = div_by(item, p.packs_magic), j = (item - i * p.packs) * V, keys = (uint32_t)p.s.keys;
  const uint32_t from = keys >= V && j + V > keys ? keys - V : j;
  k.i = i;
  k.j = from;
  k.n = (int)min((uint32_t)V, keys - from);
  k.twice = (1u << (j - from)) - 1;
  const int64_t q = p.s.d_query_pos ? p.s.d_query_pos[b * p.s.query_pos_stride + i] : p.s.query_offset + i;
  const int64_t len = p.s.d_key_lengths ? p.s.d_key_lengths[b] : p.s.keys;
  int64_t d[V];  // first keys' positions after the query, then distances
  if (p.s.d_key_pos) {
    const int64_t *kp = p.s.d_key_pos + b * p.s.key_pos_stride + from;
#pragma unroll
    for (int v = 0; v < V; v++) d[v] = kp[min(v, k.n - 1)] - q;
  } else {
#pragma unroll
    for (int v = 0; v < V; v++) d[v] = (int64_t)from + v - q;
  }
  uint32_t after = 0;
#pragma unroll
  for (int v = 0; v < V; v++) {
    after |= d[v] > 0 ? 1u << v : 0u;
    const int64_t back = -d[v];
    d[v] = d[v] > 0 ? (p.both ? d[v] : 0) : back;
    d[v] = min(d[v], INT64_MAX - 1);  // below the number behind the last threshold
    k.bucket[v] = f.reached[cell_of((uint64_t)d[v])];
  }
  for (int s = 0; s < p.steps; s++)
#pragma unroll
    for (int v = 0; v < V; v++) k.bucket[v] += d[v] >= f.threshold[k.bucket[v]];
  const int apart = p.both ? p.thresholds + 1 : 0;
  k.masked = p.s.causal ? after : 0u;
  const int64_t left = max(len, (int64_t)0) - (int64_t)from;  // keys from here that are not masked
  k.masked |= left >= V ? 0u : left <= 0 ? ~0u : ~0u << left;
  k.masked &= (1u << V) - 1;
#pragma unroll
  for (int v = 0; v < V; v++) k.bucket[v] += after >> v & 1 ? apart : 0;
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

// where a pack's keys lie (as find_keys has them), and which of them are its own
template <int V>
__device__ inline void place_of(const Shape &p, uint32_t item, uint32_t &i, uint32_t &from, uint32_t &mine) {
  const uint32_t keys = (uint32_t)p.s.keys;
  i = div_by(item, p.packs_magic);
  const uint32_t j = (item - i * p.packs) * V;
  from = keys >= V && j + V > keys ? keys - V : j;
  mine = ~((1u << (j - from)) - 1) & ((1u << min((uint32_t)V, keys - from)) - 1);
}

// PLAIN: every pack is written whole (two that overlap write the same), which spares a branch a head (16 x 2048 x 2048: 41 us, without 26).
// Not for rows shorter than a pack, nor where a pack that is read may be written already by the one that overlaps it.
// Bound by memory: 512 x 8 x 1 x 1001 in fp32 8.6 us, 256 x 4 x 199 x 199 in binary16 31 us (5.2 TB/s), 16 x 2048 x 2048 in bfloat16, written only,
// 27 us (5 TB/s).
// A workgroup has a group of heads (blockIdx.y), whose part of the table it keeps in LDS, and of all samples' packs of keys every
// gridDim.x-th 256.
template <int DT, bool SCORES, bool PLAIN>
__global__ __launch_bounds__(kThreads) void bias_forward_kernel(Shape p, int group, const void *table, int table_dtype, const typename Elem<DT>::type *scores,
                                                                tbe_bias_strides ss, float scale, float mask, typename Elem<DT>::type *out,
                                                                tbe_bias_strides os, bool in_place) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E);
  __shared__ __align__(16) Finder find;
  extern __shared__ float value[];  // [group][buckets]
  const int h0 = blockIdx.y * group, heads = min(group, p.heads - h0);
  load_finder(p, find);
  for (int k = threadIdx.x; k < heads * p.buckets; k += kThreads)
    value[k] = table_value(table, table_dtype, (int64_t)(k % p.buckets) * p.heads + h0 + k / p.buckets);
  __syncthreads();
  const bool short_row = !PLAIN && p.s.keys < V;
  const int64_t items = p.s.queries * p.packs, blocks = (items + kThreads - 1) / kThreads;
  for (int64_t w = blockIdx.x; w < blocks * p.s.batch; w += gridDim.x) {
    const int64_t b = w / blocks, item = (w - b * blocks) * kThreads + threadIdx.x;
    if (item >= items) continue;
    // The first heads' scores are asked for before the buckets are looked for.  Lanes that want nothing (keys beyond the sample's) read
    // one place, and need no branch.
    uint32_t i, j, mine;
    place_of<V>(p, (uint32_t)item, i, j, mine);
    const bool beyond = p.s.d_key_lengths && (int64_t)j >= p.s.d_key_lengths[b];
    const E *in = beyond && !short_row ? scores : scores + b * ss.sample + h0 * ss.head + i * ss.query + j;
    const int64_t step = beyond && !short_row ? 0 : ss.head;
    auto load = [&](int h, Pack<E, V>(&x)[kHeads]) {
      if (!short_row) {
#pragma unroll
        for (int g = 0; g < kHeads; g++) x[g] = read_pack<E, V>(in + min(h + g, heads - 1) * step);
      } else {
#pragma unroll
        for (int g = 0; g < kHeads; g++)
#pragma unroll
          for (int v = 0; v < V; v++) x[g].e[v] = in[min(h + g, heads - 1) * step + min(v, (int)p.s.keys - 1)];
      }
    };
    Pack<E, V> x[kHeads];
    if (SCORES) load(0, x);
    Keys<V> k;
    find_keys<V>(p, find, b, (uint32_t)item, k);
    E *to = out + b * os.sample + h0 * os.head + i * os.query + j;
    const bool whole = k.n == V && !(in_place && k.twice);  // in place: what the pack before it has is not written again
    for (int h = 0; h < heads; h += kHeads) {
      if (SCORES && h) load(h, x);
#pragma unroll
      for (int g = 0; g < kHeads; g++) {
        if (h + g >= heads) break;
        Pack<E, V> y;
#pragma unroll
        for (int v = 0; v < V; v++) {
          float r = value[(h + g) * p.buckets + k.bucket[v]];
          if (SCORES) r += (float)x[g].e[v] * scale;
          y.e[v] = (E)(k.masked >> v & 1 ? mask : r);
        }
        if (PLAIN || whole) write_pack<E, V>(to + (h + g) * os.head, y);
        else
#pragma unroll
          for (int v = 0; v < V; v++)
            if (v < k.n && !(k.twice >> v & 1)) to[(h + g) * os.head + v] = y.e[v];
      }
    }
  }
}

// Gradient of the table.  A wavefront finds the buckets of 64 packs of keys at a time and keeps those packs that are not masked altogether in
// a list in LDS.  Whenever the list has kRounds * 64 packs, it goes through the heads with them: every lane adds to sums of its own in LDS,
// [buckets + 1][64 lanes] (no two lanes on one bank; the row more takes what is masked), and the 64 lanes' sums of a head are then
// added up into the wavefront's [heads][buckets].  One lane, one order: the same bits each time.  What bounds it is the way through LDS
// and back of each addition (256 x 4 x 199 x 199, two thirds masked: 55 us), so a masked pack costs nothing here.
// (Additions by LDS atomics take several times as long, also without two lanes on one bank: 295 us instead of 81 for 256 x 4 x 199 x 199.)
constexpr int kRounds = 4, kList = (kRounds + 1) * 64;

// LDS of a wavefront, in floats
__host__ __device__ inline int grad_floats(int buckets, int group, int V) {
  return (buckets + 1) * 64 + kList * (V / 2 + 2) + ((group * buckets + 3) & ~3);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(Shape p, int group, const typename Elem<DT>::type *dout, tbe_bias_strides ds, float *part) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E);
  using Codes = Pack<uint16_t, V>;
  __shared__ __align__(16) Finder find;
  extern __shared__ __align__(16) float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64, h0 = blockIdx.y * group, heads = min(group, p.heads - h0);
  const int rows = p.buckets + 1, own = grad_floats(p.buckets, group, V);
  float *lanes = lds + wave * own;
  Codes *codes = (Codes *)(lanes + rows * 64);                   // [kList]
  int64_t *from = (int64_t *)(codes + kList);                    // [kList]: where in dout
  float *sum = (float *)(from + kList);
  load_finder(p, find);
  for (int k = threadIdx.x; k < waves * own; k += blockDim.x) lds[k] = 0.0f;
  __syncthreads();
  const uint32_t items = (uint32_t)(p.s.queries * p.packs), steps = (items + 63) / 64;
  const bool short_row = p.s.keys < V;
  int width = 1;  // 64 / width lanes add up a row of lanes' sums
  while (width < p.buckets && width < 64) width *= 2;

  auto load = [&](int h, Pack<E, V>(&x)[kRounds]) {
    const E *in = dout + (h0 + h) * ds.head;
    if (!short_row) {
#pragma unroll
      for (int r = 0; r < kRounds; r++) x[r] = read_pack<E, V>(in + from[r * 64 + lane]);
    } else {
#pragma unroll
      for (int r = 0; r < kRounds; r++)
#pragma unroll
        for (int v = 0; v < V; v++) x[r].e[v] = in[from[r * 64 + lane] + min(v, (int)p.s.keys - 1)];
    }
  };
  // the first n packs of the list, through all heads
  auto through_heads = [&](int n) {
    for (int k = n + lane; k < kRounds * 64; k += 64) {  // places that no pack has taken
      Codes c;
#pragma unroll
      for (int v = 0; v < V; v++) c.e[v] = (uint16_t)p.buckets;
      codes[k] = c;
      from[k] = 0;
    }
    __builtin_amdgcn_wave_barrier();
    Pack<E, V> x[kRounds], next[kRounds];
    load(0, next);
#pragma unroll 1
    for (int h = 0; h < heads; h++) {
#pragma unroll
      for (int r = 0; r < kRounds; r++) x[r] = next[r];
      if (h + 1 < heads) load(h + 1, next);
#pragma unroll
      for (int r = 0; r < kRounds; r++) {
        if (r * 64 >= n) break;  // the same in all lanes
        const Codes c = codes[r * 64 + lane];
#pragma unroll
        for (int v = 0; v < V; v++) lanes[c.e[v] * 64 + lane] += (float)x[r].e[v];
      }
      // lanes' sums of this head, and zeros for the next one's (the row of what is masked may hold anything)
      for (int c0 = 0; c0 < p.buckets; c0 += width) {
        const int c = c0 + (lane & (width - 1));
        float v = 0.0f;
        if (c < p.buckets)
#pragma unroll 8
          for (int k = lane / width; k < 64; k += 64 / width) {
            float *q = lanes + c * 64 + ((k + c) & 63);
            v += *q;
            *q = 0.0f;
          }
        for (int k = width; k < 64; k *= 2) v += __shfl_xor(v, k);
        if (c < p.buckets && lane < width) sum[h * p.buckets + c] += v;
      }
      __builtin_amdgcn_wave_barrier();
    }
  };

  int n = 0;  // packs in the list
  for (int64_t w = (int64_t)blockIdx.x * waves + wave; w < steps * p.s.batch; w += (int64_t)gridDim.x * waves) {
    const int64_t b = w / steps;
    const uint32_t item = (uint32_t)(w - b * steps) * 64 + lane;
    Keys<V> k;
    find_keys<V>(p, find, b, min(item, items - 1), k);
    const uint32_t mine = item < items ? ~k.twice & ((1u << k.n) - 1) : 0u, out = k.masked | ~mine;
    Codes c;
    bool any = false;
#pragma unroll
    for (int v = 0; v < V; v++) {
      c.e[v] = (uint16_t)(out >> v & 1 ? p.buckets : k.bucket[v]);
      any |= c.e[v] != p.buckets;
    }
    const uint64_t listed = __ballot(any);
    if (any) {
      const int at = n + __popcll(listed & ((1ull << lane) - 1));
      codes[at] = c;
      from[at] = b * ds.sample + k.i * ds.query + k.j;
    }
    n += __popcll(listed);
    __builtin_amdgcn_wave_barrier();
    if (n >= kRounds * 64) {
      through_heads(kRounds * 64);
      n -= kRounds * 64;
      if (lane < n) {  // what the list had more is its beginning now
        codes[lane] = codes[kRounds * 64 + lane];
        from[lane] = from[kRounds * 64 + lane];
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  if (n) through_heads(n);
  __syncthreads();
  for (int k = threadIdx.x; k < heads * p.buckets; k += blockDim.x) {
    float v = 0.0f;
    for (int w = 0; w < waves; w++) v += lds[(w + 1) * own - ((group * p.buckets + 3) & ~3) + k];
    part[((int64_t)blockIdx.x * p.heads + h0) * p.buckets + k] = v;
  }
}

// Gradient of the scores where positions are given: an element at a time, after the table's (in place it may take d_dout's place).
template <int DT>
__global__ __launch_bounds__(kThreads) void bias_scores_kernel(Shape p, const typename Elem<DT>::type *dout, tbe_bias_strides ds, float scale,
                                                               typename Elem<DT>::type *dscores, tbe_bias_strides es) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E);
  const int64_t items = p.s.queries * p.packs, blocks = (items + kThreads - 1) / kThreads;
  for (int64_t w = blockIdx.x; w < blocks * p.s.batch; w += gridDim.x) {
    const int64_t b = w / blocks, item = (w - b * blocks) * kThreads + threadIdx.x;
    if (item >= items) continue;
    const int64_t i = (int64_t)div_by((uint32_t)item, p.packs_magic), j = (item - i * p.packs) * V;
    const int64_t q = p.s.d_query_pos ? p.s.d_query_pos[b * p.s.query_pos_stride + i] : p.s.query_offset + i;
    const int64_t len = p.s.d_key_lengths ? p.s.d_key_lengths[b] : p.s.keys;
    const int n = (int)min((int64_t)V, p.s.keys - j);
    uint32_t keep = 0;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int64_t at = j + min(v, n - 1), pos = p.s.d_key_pos ? p.s.d_key_pos[b * p.s.key_pos_stride + at] : at;
      const bool later = p.s.causal && pos > q, beyond = j + v >= len;
      keep |= (later | beyond) ? 0u : 1u << v;
    }
    for (int h = 0; h < p.heads; h++) {
      const E *in = dout + b * ds.sample + h * ds.head + i * ds.query + j;
      E *to = dscores + b * es.sample + h * es.head + i * es.query + j;
      Pack<E, V> x;
      if (n == V) x = read_pack<E, V>(in);
      else
#pragma unroll
        for (int v = 0; v < V; v++) x.e[v] = in[min(v, n - 1)];
#pragma unroll
      for (int v = 0; v < V; v++) x.e[v] = (E)(keep >> v & 1 ? (float)x.e[v] * scale : 0.0f);
      if (n == V) write_pack<E, V>(to, x);
      else
#pragma unroll
        for (int v = 0; v < V; v++)
          if (v < n) to[v] = x.e[v];
    }
  }
}

// The same where positions are indices: then a bucket is a matter of key - query, of the diagonal.  A lane takes squares of V keys by V queries
// one after another down a diagonal, which all have the same 2 V - 1 diagonals, and keeps their sums in registers: one addition an element,
// and every load a whole pack.  64 lanes have neighbouring squares.  A wavefront's unit of work is 64 such columns of squares, `seg`
// squares of each (of the same queries), for `samples` samples; at its end its diagonals are joined in LDS and added to their buckets.
// Bound by the latency of memory, with four wavefronts a SIMD: 16 x 8 x 1024 x 1024 in bfloat16 52 us (5.1 TB/s) where the cache holds the
// scores, 60 where not; by the kernel above 140.
constexpr int kUnits = 4096;  // units that the work is cut into, if they have 4 squares at least (16 x 8 x 1024 x 1024: 52 us; 8192: 65)

struct Diagonals {
  uint32_t squares;       // of V queries
  uint32_t columns, segs, batches;  // units of a head
  int seg, samples;
  bool band;              // columns are counted from the first one that a segment's squares lie in (few keys: most have nothing of it)
};

template <int DT, bool SCORES>
__global__ __launch_bounds__(kThreads, SCORES ? 2 : 4) void bias_grad_index_kernel(Shape p, Diagonals u, const typename Elem<DT>::type *dout, tbe_bias_strides ds,
                                                                   float *part, float scale, typename Elem<DT>::type *dscores, tbe_bias_strides es) {
  using E = typename Elem<DT>::type;
  constexpr int V = 16 / sizeof(E), kDiagonals = 64 * V + V - 1;
  __shared__ __align__(16) Finder find;
  __shared__ float diagonals[kWaves][kDiagonals + 1];
  extern __shared__ float sums[];  // [kWaves][buckets]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y;
  float *diag = diagonals[wave], *sum = sums + wave * p.buckets;
  load_finder(p, find);
  for (int k = threadIdx.x; k < kWaves * p.buckets; k += kThreads) sums[k] = 0.0f;
  __syncthreads();
  const int keys = (int)p.s.keys, queries = (int)p.s.queries, packs = (int)p.packs, squares = (int)u.squares;
  const int64_t units = (int64_t)u.columns * u.segs * u.batches;
  const bool short_row = keys < V;
  for (int64_t w = (int64_t)blockIdx.x * kWaves + wave; w < units; w += (int64_t)gridDim.x * kWaves) {
    const int s = (int)(w / u.columns % u.segs);
    const int column = (int)(w % u.columns) + (u.band ? (squares - min((s + 1) * u.seg, squares)) / 64 : 0);
    const int64_t b0 = w / u.columns / u.segs * u.samples, b1 = min(b0 + u.samples, p.s.batch);
    const int first = 64 * column - (squares - 1), D = first + lane;  // key square less query square
    const int lo = max(s * u.seg, -(first + 63)), hi = min(min((s + 1) * u.seg, squares), packs - first);
    if (lo >= hi) continue;
    const bool later = p.s.causal && (int64_t)D * V - (V - 1) - p.s.query_offset > 0;  // all of them masked
    float acc[2 * V - 1];
#pragma unroll
    for (int k = 0; k < 2 * V - 1; k++) acc[k] = 0.0f;
    for (int64_t b = b0; b < b1; b++) {
      // at most the keys: a short row's places beyond them hold its last key again
      const int64_t len = p.s.d_key_lengths ? max(min(p.s.d_key_lengths[b], p.s.keys), (int64_t)0) : p.s.keys;
      const E *in = dout + b * ds.sample + h * ds.head;
      for (int q = lo; q < hi; q++) {
        const int j = (int)((uint32_t)(q + D) * V), i = q * V;  // j where `on`
        const bool on = q + D >= 0 && q + D < packs;
        const int left = (int)max(min(len - j, (int64_t)V), (int64_t)0);  // keys that are not beyond the sample's
        if (!on || (!SCORES && (later || left == 0))) continue;
        Pack<E, V> x[V];
        const int back = keys - j < V ? V - (keys - j) : 0;  // places of the last pack that are beyond the row (j + V may be 2^31)
        const E *from = in + (int64_t)i * ds.query + j - (short_row ? 0 : back);
        const int64_t last = (int64_t)min(V, queries - i) - 1;
        if (!short_row) {
#pragma unroll
          for (int r = 0; r < V; r++) x[r] = read_pack<E, V>(from + min((int64_t)r, last) * ds.query);
          if (back)  // that pack ends where the row does: down with it
#pragma unroll
            for (int r = 0; r < V; r++) {
              uint64_t v[2];
              __builtin_memcpy(v, &x[r], 16);
              const int bits = back * 8 * (int)sizeof(E);
              const uint64_t lo = bits >= 64 ? v[1] >> (bits - 64) : v[0] >> bits | v[1] << (64 - bits);
              v[1] = bits >= 64 ? 0 : v[1] >> bits;
              v[0] = lo;
              __builtin_memcpy(&x[r], v, 16);
            }
        } else {
#pragma unroll
          for (int r = 0; r < V; r++)
#pragma unroll
            for (int v = 0; v < V; v++) x[r].e[v] = from[min((int64_t)r, last) * ds.query + min(v, keys - 1)];
        }
        const int rows = queries - i;
        if (left < V || rows < V)
#pragma unroll
          for (int r = 0; r < V; r++)
#pragma unroll
            for (int v = 0; v < V; v++) x[r].e[v] = v < left && r < rows ? x[r].e[v] : (E)0.0f;
#pragma unroll
        for (int r = 0; r < V; r++) {
#pragma unroll
          for (int v = 0; v < V; v++) {
            const float g = (float)x[r].e[v];
            acc[V - 1 + v - r] += g;
            if (SCORES) x[r].e[v] = (E)(p.s.causal && (int64_t)D * V + v - r - p.s.query_offset > 0 ? 0.0f : g * scale);
          }
          if (SCORES && r < rows) {
            E *to = dscores + b * es.sample + h * es.head + (int64_t)(i + r) * es.query + j;
            if (!back) write_pack<E, V>(to, x[r]);
            else
#pragma unroll
              for (int v = 0; v < V; v++)
                if (j + v < keys) to[v] = x[r].e[v];
          }
        }
      }
    }
    // diag[k]: diagonal first * V - (V - 1) + k.  A lane's upper V diagonals first, then its lower ones to the upper ones of the lane before
#pragma unroll
    for (int k = 0; k < V; k++) diag[lane * V + V - 1 + k] = acc[V - 1 + k];
    if (lane < V - 1) diag[lane] = 0.0f;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < V - 1; k++) diag[lane * V + k] += acc[k];
    __builtin_amdgcn_wave_barrier();
    for (int k0 = 0; k0 < kDiagonals; k0 += 64) {
      const int64_t ahead = (int64_t)first * V - (V - 1) + k0 + lane - p.s.query_offset;
      const bool there = k0 + lane < kDiagonals && !(p.s.causal && ahead > 0);
      const int c = bucket_of(p, find, ahead);
      const float v = there ? diag[k0 + lane] : 0.0f;
      uint64_t todo = __ballot(there);
      while (todo) {  // a bucket at a time: one, unless the diagonals are near
        const int one = __shfl(c, __ffsll((unsigned long long)todo) - 1);
        const bool mine = there && c == one;
        float r = mine ? v : 0.0f;
        for (int k = 32; k; k >>= 1) r += __shfl_xor(r, k);
        if (lane == 0) sum[one] += r;
        todo &= ~__ballot(mine);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  for (int k = threadIdx.x; k < p.buckets; k += kThreads) {
    float v = 0.0f;
    for (int w = 0; w < kWaves; w++) v += sums[w * p.buckets + k];
    part[((int64_t)blockIdx.x * p.heads + h) * p.buckets + k] = v;
  }
}

// A wavefront for each number of the table's gradient; 5 us for up to 1024 sums of each.
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
  int steps = 1;
  bool both = false;
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
  *out = {*p, s->heads, s->thresholds, s->buckets, s->both, s->steps, s->map, packs, div_magic(packs)};
  return TBE_OK;
}

// whether two sets of strides name the same places (those of a single sample, head or query name none)
bool same_places(const Shape &p, const tbe_bias_strides &a, const tbe_bias_strides &b) {
  return (p.s.batch < 2 || a.sample == b.sample) && (p.heads < 2 || a.head == b.head) && (p.s.queries < 2 || a.query == b.query);
}

int64_t blocks_of(const Shape &p) { return (p.s.queries * p.packs + kThreads - 1) / kThreads * p.s.batch; }

}  // namespace

extern "C" {

int tbe_bias_destroy(tbe_bias_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->map);
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
  int all = 0, some = 0;                // thresholds up to lo and hi
  for (int c = 0; c < kCells; c++) {  // distances lo .. hi can lie in the cell; the next cell's border is hi + 1
    int64_t lo = 0, hi = 0;
    if (c > 0) {
      const double from = border_of(c), to = border_of(c + 1), below = from >= 4194304.0 ? from * (1.0 - 0x1p-22) : from;
      lo = below >= 0x1p63 ? INT64_MAX - 1 : (int64_t)std::ceil(below);
      hi = to >= 0x1p63 ? INT64_MAX - 1 : (int64_t)std::ceil(to) - 1;
    }
    while (all < num_thresholds && h_thresholds[all] <= lo) all++;
    while (some < num_thresholds && h_thresholds[some] <= hi) some++;
    map.reached[c] = (uint8_t)all;
    if (some - all > s->steps) s->steps = some - all;
  }
  hipError_t e = hipGetDevice(&s->device);  // one block: [map][part]
  if (e == hipSuccess) e = hipMalloc((void **)&s->map, sizeof(Buckets) + (size_t)kMaxParts * heads * s->buckets * sizeof(float));
  s->part = (float *)(s->map + 1);
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
  if (d_out == d_scores && !same_places(p, ss, *out_strides)) return report(TBE_EINVAL, "in place with other strides");
  const int group = p.heads < kTableFloats / p.buckets ? p.heads : kTableFloats / p.buckets, groups = (p.heads + group - 1) / group;
  const int64_t blocks = blocks_of(p);
  const dim3 grid((unsigned)(blocks < kForward ? blocks : kForward), (unsigned)groups);
  const size_t lds = (size_t)group * p.buckets * sizeof(float);
  const int V = 16 / elem_bytes(p.s.dtype);
  const bool plain = p.s.keys >= V && (p.s.keys % V == 0 || d_out != d_scores);
#define LAUNCH(DT, SCORES, PLAIN)                                                                                                       \
  bias_forward_kernel<DT, SCORES, PLAIN><<<grid, kThreads, lds, (hipStream_t)stream>>>(p, group, d_table, table_dtype, (const Elem<DT>::type *)d_scores, ss, \
                                                                                scale, mask_value, (Elem<DT>::type *)d_out, *out_strides, d_out == d_scores)
#define LAUNCH2(DT)                                                   \
  (d_scores ? plain ? LAUNCH(DT, true, true) : LAUNCH(DT, true, false) \
            : plain ? LAUNCH(DT, false, true) : LAUNCH(DT, false, false))
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
  const tbe_bias_strides es = any && d_dscores ? *dscores_strides : tbe_bias_strides{0, 0, 0};
  if (any && d_dscores == d_dout && !same_places(p, *dout_strides, es)) return report(TBE_EINVAL, "in place with other strides");
  int parts = 0;
  if (any) {
    if (!p.s.d_query_pos && !p.s.d_key_pos) {
      // Units long enough that joining their diagonals does not count, and enough of them for all CUs.
      const int V = 16 / elem_bytes(p.s.dtype);
      Diagonals u;
      u.squares = (uint32_t)((p.s.queries + V - 1) / V);
      const uint32_t columns = (u.squares + p.packs - 1 + 63) / 64;
      const int64_t squares = (int64_t)columns * u.squares * p.s.batch * p.heads;  // times 64, some of them beyond the scores
      const int64_t steps = squares / kUnits < 4 ? 4 : squares / kUnits > 64 ? 64 : squares / kUnits;
      u.seg = (int)(steps < u.squares ? steps : u.squares);
      u.segs = (u.squares + u.seg - 1) / u.seg;
      // A segment's squares lie on packs + seg - 1 neighbouring diagonals, the units on all columns would grow with the queries' square.
      const uint32_t band = (p.packs + u.seg - 2 + 63) / 64 + 1;
      u.band = band <= columns / 2;
      u.columns = u.band ? band : columns;
      const int64_t samples = steps / u.seg;
      u.samples = (int)(samples < p.s.batch ? samples : p.s.batch);
      u.batches = (uint32_t)((p.s.batch + u.samples - 1) / u.samples);
      const int64_t units = (int64_t)u.columns * u.segs * u.batches, blocks = (units + kWaves - 1) / kWaves;
      parts = (int)(blocks < kMaxParts ? blocks : kMaxParts);
      const dim3 grid((unsigned)parts, (unsigned)p.heads);
      const size_t lds = (size_t)kWaves * p.buckets * sizeof(float);
#define LAUNCH(DT, SCORES)                                                                                                                    \
  bias_grad_index_kernel<DT, SCORES><<<grid, kThreads, lds, (hipStream_t)stream>>>(p, u, (const Elem<DT>::type *)d_dout, *dout_strides, s->part, scale, \
                                                                                   (Elem<DT>::type *)d_dscores, es)
#define LAUNCH2(DT) (d_dscores ? LAUNCH(DT, true) : LAUNCH(DT, false))
      if (p.s.dtype == TBE_FP32) LAUNCH2(TBE_FP32);
      else if (p.s.dtype == TBE_FP16) LAUNCH2(TBE_FP16);
      else LAUNCH2(TBE_BF16);
#undef LAUNCH2
#undef LAUNCH
    } else {
      // heads of a workgroup: all, unless their sums take more than 8 KB of a wavefront, or there are too few packs to fill the GPU
      const int64_t steps = (p.s.queries * p.packs + 63) / 64 * p.s.batch, lists = (steps + kRounds - 1) / kRounds;
      int group = p.heads;
      while (group > 1 && group * p.buckets > kSums) group = (group + 1) / 2;
      while (group > 1 && lists * ((p.heads + group - 1) / group) < kFill) group = (group + 1) / 2;
      // wavefronts of a workgroup: as many as have room for their sums beside the finder
      const size_t own = grad_floats(p.buckets, group, 16 / elem_bytes(p.s.dtype)) * sizeof(float);
      const int waves = 4 * own + sizeof(Finder) <= kLds ? 4 : 3 * own + sizeof(Finder) <= kLds ? 3 : 2 * own + sizeof(Finder) <= kLds ? 2 : 1;
      parts = (int)((lists + waves - 1) / waves < kMaxParts ? (lists + waves - 1) / waves : kMaxParts);
      const dim3 grid((unsigned)parts, (unsigned)((p.heads + group - 1) / group));
      const size_t lds = waves * own;
      const int64_t blocks = blocks_of(p);
      const dim3 all((unsigned)(blocks < 4096 ? blocks : 4096));
#define LAUNCH2(DT)                                                                                                                              \
  do {                                                                                                                                           \
    if (d_dtable)                                                                                                                                \
      bias_grad_kernel<DT><<<grid, 64 * waves, lds, (hipStream_t)stream>>>(p, group, (const Elem<DT>::type *)d_dout, *dout_strides, s->part);    \
    if (d_dscores)                                                                                                                               \
      bias_scores_kernel<DT><<<all, kThreads, 0, (hipStream_t)stream>>>(p, (const Elem<DT>::type *)d_dout, *dout_strides, scale,                 \
                                                                        (Elem<DT>::type *)d_dscores, es);                                        \
  } while (0)
      if (p.s.dtype == TBE_FP32) LAUNCH2(TBE_FP32);
      else if (p.s.dtype == TBE_FP16) LAUNCH2(TBE_FP16);
      else LAUNCH2(TBE_BF16);
    }
#undef LAUNCH2
  }
  if (d_dtable)
    bias_join_kernel<<<dim3((unsigned)((p.heads * p.buckets + kWaves - 1) / kWaves)), kThreads, 0, (hipStream_t)stream>>>(s->part, parts, p.heads,
                                                                                                                        p.buckets, d_dtable);
  return check_launch();
}

}  // extern "C"
