// Short causal convolution over the rows of every bag: forward, backward, one row for each of many states.
// Contract: include/tbe.h.
//
//   v_t = bias + sum over j < W of w_j e_{t-W+1+j},  e: a bag's earlier rows and its rows;  y = v or silu(v).
//   With g = dy silu'(v):  de_i = sum over k < W of w_{W-1-k} g_{i+k} (rows of the bag),  dw_j = sum over t of g_t e_{t-W+1+j},  dbias = sum of g.
//
// Rows in fp32 are bound by memory, rows in 16 bits by vector instructions (0.8 of the forward's time, 0.65 of the backward's).  A workgroup takes a tile of rows wherever bags begin; a lane walks V elements of so many rows in a row down, all of which it reads
// at first, and W - 1 in front of them once more (from the caches).  Where bags start within the tile is written to LDS meanwhile.  Rows
// near a bag's start, which do not see all of the rows in front of them, take a way of their own.  The backward walks the same way and
// W - 1 rows on: it finds v again, keeps the sums of the last W rows' gradients and gives a row up when the last result that sees it is done.
// 245760 rows of 128 in bags of 30, bfloat16, width 4 with silu: forward 36 us (3.5 TB/s), backward
// 79 us (146 when rows were read one by one), in fp32 56 (4.5 TB/s) and 137 us; three bags of 100 k rows of 64, fp32, width 3: 29 us (packs of 16 bytes 33).
#include <algorithm>
#include <new>

#include "tbe_rows.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 8;                   // of a lane in a tile
constexpr int grad_rows(int width) { return width <= 4 ? 8 : 4; }  // ... in the backward: its lanes hold those that see them too
constexpr int kMostWidth = 8;
constexpr int64_t kMostParts = 1024;       // workgroups of the backward, each with partial sums of dw and dbias

struct ConvArgs {
  const void *x, *weight, *bias, *before, *dy, *dlast;
  int64_t xs, ys, dys, dxs, rows, bags;
  const int64_t *off;
  void *y, *last, *dx, *dbefore;
  float *parts;
  int dim, lanes, passes, weight_dtype;
  int64_t tiles, first_group;
  int32_t *err;
  bool silu;
};

template <class E> constexpr int kPack = 8 / sizeof(E);
template <class E> constexpr int kGradPack = 8 / sizeof(E);

// Bags that start in rows [r0, r1): marks[row - r0] = bag, -1 elsewhere; head: the bag that row r0 belongs to and its first row
struct Head {
  int64_t bag, start;
};
__device__ inline Head mark_tile(const ConvArgs &a, int64_t r0, int64_t r1, int *marks, int count) {
  for (int i = threadIdx.x; i < count; i += kThreads) marks[i] = -1;
  const int64_t lo = count_up_to(a.off, a.bags, r0), head = max(lo - 1, (int64_t)0);
  __syncthreads();
  for (int64_t b = head + threadIdx.x; b < a.bags; b += kThreads) {
    const int64_t s = a.off[b], e = a.off[b + 1];
    if (s >= r1) break;
    if (s >= r0 && e > s) marks[s - r0] = (int)b;
  }
  __syncthreads();
  return {head, min(a.off[head], r0)};
}

// how many rows of its bag row r, the first of a walk, has in front of it, W - 1 or more as W - 1, and its bag if there are fewer
template <int W>
__device__ inline int age_of(const int *marks, int64_t r0, int64_t r, Head head, int64_t &bag) {
  bag = head.bag;
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    if (r - k < r0) break;
    if (marks[r - k - r0] >= 0) {
      bag = marks[r - k - r0];
      return k;
    }
  }
  return (int)min(max(r - head.start, (int64_t)0), (int64_t)(W - 1));
}

// Where a bag has only `age` < W - 1 rows in front of one, the others that its result and those after it see are earlier ones, or zero.
template <class E, int W, int V>
__device__ inline void young(const ConvArgs &a, int age, int64_t bag, int at, int n, float (&e)[W][V]) {
#pragma unroll
  for (int k = 0; k < W - 1; ++k)  // e[k]: W - 1 - k rows back
    if (W - 1 - k > age) {
      if (a.before) {
        load_floats<E, V>((const E *)a.before + (bag * (W - 1) + k + age) * a.dim + at, n, e[k]);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) e[k][j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) asm volatile("" : "+v"(e[k][j]));  // waited for here, and not by the rows that load nothing
    }
}

// The weights of V elements lie one behind another: one look at their type, wide loads.  (A look for each was a wait for each, 20 of them.)
template <int W, int V>
__device__ inline void load_weights(const ConvArgs &a, int at, float (&w)[W][V], float (&bias)[V]) {
  float all[V * W];
  load_params<V * W>(a.weight, a.weight_dtype, (int64_t)at * W, (a.dim - at) * W, all);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    bias[j] = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k][j] = all[j * W + k];
  }
  if (a.bias) load_params<V>(a.bias, a.weight_dtype, at, a.dim - at, bias);
}

template <int W, int V, class R>
__device__ inline void next_row(float (&e)[W][V], const R &x) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int k = 0; k < W - 1; ++k) e[k][j] = e[k + 1][j];
    e[W - 1][j] = x.get(j);
  }
}
template <int W, int V>
__device__ inline void result(const float (&e)[W][V], const float (&w)[W][V], const float (&bias)[V], float (&v)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    v[j] = bias[j];
#pragma unroll
    for (int k = 0; k < W; ++k) v[j] += w[k][j] * e[k][j];
  }
}

// whether bag b has offsets that do not ascend from 0 to rows, which are reported
__device__ inline bool refused(const ConvArgs &a, int64_t b, int64_t s, int64_t e, bool say) {
  const bool bad = s > e || s < 0 || e > a.rows || (b == 0 && s != 0) || (b == a.bags - 1 && e != a.rows);
  if (bad && say) *a.err = 1;
  return bad;
}
// The lanes behind the tiles have a pack each of a row m of what is a bag's own: of its last W - 1 rows, from the rows or the earlier ones
template <class E, int W>
__device__ inline void last_rows(const ConvArgs &a, int64_t i) {
  if constexpr (W > 1) {
    constexpr int V = kPack<E>;
    const int packs = (a.dim + V - 1) / V;
    const int64_t row = quotient(i, packs), b = quotient(row, W - 1);
    if (b >= a.bags) return;
    const int m = (int)(row - b * (W - 1)), at = (int)(i - row * packs) * V;
    const int64_t s = a.off[b], e = a.off[b + 1];
    if (refused(a, b, s, e, m == 0 && at == 0)) return;
    const int64_t r = e - (W - 1) + m;
    Words<E, V> v;
    if (r >= s) load_words<E, V>((const E *)a.x + r * a.xs + at, a.dim - at, v);
    else if (a.before) load_words<E, V>((const E *)a.before + (b * (W - 1) + r - s + W - 1) * a.dim + at, a.dim - at, v);
    else v = {};
    store_words<E, V>((E *)a.last + row * a.dim + at, a.dim - at, v);
  }
}
// or, in the backward, an element of the gradient of the earlier rows: sum over t <= m of w_{m-t} g_t, and what of dlast goes past the bag's rows
template <class E, int W>
__device__ inline void earlier_rows(const ConvArgs &a, int64_t i) {
  if constexpr (W > 1) {
    const int64_t row = quotient(i, a.dim), b = quotient(row, W - 1);
    if (b >= a.bags) return;
    const int m = (int)(row - b * (W - 1)), d = (int)(i - row * a.dim);
    const int64_t s = a.off[b], e = a.off[b + 1], size = e - s;
    if (refused(a, b, s, e, m == 0 && d == 0)) return;
    float sum = a.dlast && m >= size ? (float)((const E *)a.dlast)[(row - size) * a.dim + d] : 0.0f;
    for (int t = 0; t <= m && t < size; ++t) {
      float g = (float)((const E *)a.dy)[(s + t) * a.dys + d];
      if (a.silu) {
        float v = a.bias ? load_param(a.bias, a.weight_dtype, d) : 0.0f;
        for (int k = 0; k < W; ++k) {
          const int back = W - 1 - k;
          const float x = back <= t ? (float)((const E *)a.x)[(s + t - back) * a.xs + d]
                                    : a.before ? (float)((const E *)a.before)[(b * (W - 1) + t + k) * a.dim + d] : 0.0f;
          v += load_param(a.weight, a.weight_dtype, (int64_t)d * W + k) * x;
        }
        const float f = sigmoid(v);
        g *= f * (1.0f + v * (1.0f - f));
      }
      sum += load_param(a.weight, a.weight_dtype, (int64_t)d * W + m - t) * g;
    }
    ((E *)a.dbefore)[i] = (E)sum;
  }
}
// the same look at the offsets where there are no such lanes
__device__ inline void look_over(const ConvArgs &a, int64_t b) {
  if (b < a.bags) refused(a, b, a.off[b], a.off[b + 1], true);
}

template <class E, int W>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvArgs a) {
  constexpr int V = kPack<E>;
  extern __shared__ int marks[];
  const int64_t group = a.first_group + blockIdx.x;
  if (group >= a.tiles * a.passes) {
    const int64_t i = (group - a.tiles * a.passes) * kThreads + threadIdx.x;
    if (W > 1 && a.last) last_rows<E, W>(a, i);
    else look_over(a, i);
    return;
  }
  const int64_t tile = group / a.passes;
  const int walks = kThreads / a.lanes, tile_rows = walks * kRows;
  const int64_t r0 = tile * tile_rows, r1 = min(r0 + tile_rows, a.rows);
  const int at = ((int)(group % a.passes) * a.lanes + (threadIdx.x & (a.lanes - 1))) * V, n = a.dim - at;
  const int64_t first = r0 + threadIdx.x / a.lanes * kRows;
  const bool some = n > 0 && first < r1;
  Words<E, V> raw[W - 1 + kRows];  // rows first - (W - 1) and on
  if (some) {
#pragma unroll
    for (int i = 0; i < W - 1 + kRows; ++i) load_words<E, V>((const E *)a.x + min(max(first - (W - 1) + i, (int64_t)0), r1 - 1) * a.xs + at, n, raw[i]);
  }
  const Head head = mark_tile(a, r0, r1, marks, tile_rows);
  if (!some) return;
  float w[W][V], bias[V];
  load_weights<W, V>(a, at, w, bias);
  int64_t bag;
  int age = age_of<W>(marks, r0, first, head, bag);
  E *y = (E *)a.y + first * a.ys + at;
  const int rows = (int)min((int64_t)kRows, r1 - first);
  const int *mark = marks + (first - r0);
  float e[W][V];  // what a result sees, oldest first
#pragma unroll
  for (int k = 0; k < W - 1; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) e[k + 1][j] = raw[k].get(j);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (i >= rows) continue;
    __builtin_amdgcn_sched_barrier(0);  // rows become fp32 one by one: all at once they do not fit the registers
    next_row<W, V>(e, raw[W - 1 + i]);
    if (i > 0 && mark[i] >= 0) age = 0, bag = mark[i];
    if (i > 0 ? mark[i] >= 0 : age < W - 1) young<E, W, V>(a, age, bag, at, n, e);
    float v[V];
    result<W, V>(e, w, bias, v);
    if (a.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= sigmoid(v[j]);
    }
    store_floats<E, V>(y, n, v);
    y += a.ys;
  }
}

template <class E, int W>
__global__ __launch_bounds__(kThreads) void conv_grad_kernel(ConvArgs a, int64_t workers) {
  constexpr int V = kGradPack<E>, R = grad_rows(W), K = W + 1;  // sums of an element: W of dw, one of dbias
  extern __shared__ int marks[];                             // tile_rows + W - 1 of them, and then the sums of the walks
  const int64_t group = a.first_group + blockIdx.x;
  if (group >= workers * a.passes) {
    const int64_t i = (group - workers * a.passes) * kThreads + threadIdx.x;
    if (W > 1 && a.dbefore) earlier_rows<E, W>(a, i);
    else look_over(a, i);
    return;
  }
  const int lane = threadIdx.x & (a.lanes - 1), walk = threadIdx.x / a.lanes, walks = kThreads / a.lanes, tile_rows = walks * R;
  const int64_t worker = blockIdx.x / a.passes;  // (they are all in the first launch)
  const int at = ((int)(blockIdx.x % a.passes) * a.lanes + lane) * V, n = a.dim - at;
  float w[W][V], bias[V], dw[K][V];
  if (n > 0) load_weights<W, V>(a, at, w, bias);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[k][j] = 0.0f;
  for (int64_t tile = worker; tile < a.tiles; tile += workers) {
    const int64_t r0 = tile * tile_rows, r1 = min(r0 + tile_rows, a.rows);
    const int64_t first = r0 + walk * R, stop = min(r1 + W - 1, a.rows);
    const bool some = n > 0 && first < r1;
    Words<E, V> raw[2 * (W - 1) + R], raw_dy[W - 1 + R];  // rows first - (W - 1) and on, rows first and on
    if (some) {
#pragma unroll
      for (int i = 0; i < 2 * (W - 1) + R; ++i) load_words<E, V>((const E *)a.x + min(max(first - (W - 1) + i, (int64_t)0), stop - 1) * a.xs + at, n, raw[i]);
#pragma unroll
      for (int i = 0; i < W - 1 + R; ++i) load_words<E, V>((const E *)a.dy + min(first + i, stop - 1) * a.dys + at, n, raw_dy[i]);
    }
    __syncthreads();  // the marks of the tile before
    const Head head = mark_tile(a, r0, stop, marks, tile_rows + W - 1);
    if (!some) continue;
    int64_t bag;
    int age = age_of<W>(marks, r0, first, head, bag);
    const int *mark = marks + (first - r0);
    float e[W][V];    // what a result sees, oldest first
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) e[k + 1][j] = raw[k].get(j);
    float acc[W][V];  // acc[k]: what row t - k has had so far
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[k][j] = 0.0f;
#pragma unroll
    for (int i = 0; i < R + W - 1; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      const int64_t t = first + i;
      const bool there = t < a.rows;  // behind the last row nothing sees anything, like behind the end of a bag
      const int b = there ? mark[i] : 0;
      if (i > 0) {
        age = b >= 0 ? 0 : min(age + 1, W - 1);
        bag = b >= 0 ? b : bag;
      }
      next_row<W, V>(e, raw[W - 1 + i]);
      if (!there) age = 0;
      if (there) {
        float g[V], v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = raw_dy[i].get(j);
        if (i > 0 ? b >= 0 : age < W - 1) young<E, W, V>(a, age, bag, at, n, e);
        if (a.silu) {
          result<W, V>(e, w, bias, v);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float f = sigmoid(v[j]);
            g[j] *= f * (1.0f + v[j] * (1.0f - f));
          }
        }
        if (i < R && t < r1) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
#pragma unroll
            for (int k = 0; k < W; ++k) dw[k][j] += g[j] * e[k][j];
            dw[W][j] += g[j];
          }
        }
        if (age < W - 1) {  // only rows of its bag
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[k][j] += k <= age ? w[W - 1 - k][j] * g[j] : 0.0f;
        } else {
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[k][j] += w[W - 1 - k][j] * g[j];
        }
      }
      // row t - (W - 1) has all of its gradient but dlast's part, which rows W - 1 or less before the bag's end have
      const int64_t p = t - (W - 1);
      if (i >= W - 1 && p < r1) {
        if (age < W - 1 && a.dlast) {
          int64_t ends = stop, of = head.bag;  // (stop: all rows there are, or p is not near the end)
          for (int k = W - 1; k >= 1; --k)
            if (p + k < stop && marks[p + k - r0] >= 0) ends = p + k;
          for (int64_t r = p; r >= r0; --r)
            if (marks[r - r0] >= 0) {
              of = marks[r - r0];
              break;
            }
          float d[V];
          load_floats<E, V>((const E *)a.dlast + (of * (W - 1) + max(p - ends + W - 1, (int64_t)0)) * a.dim + at, n, d);
#pragma unroll
          for (int j = 0; j < V; ++j) acc[W - 1][j] += d[j];
        }
        store_floats<E, V>((E *)a.dx + p * a.dxs + at, n, acc[W - 1]);
      }
#pragma unroll
      for (int k = W - 1; k >= 1; --k)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] = acc[k - 1][j];
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = 0.0f;
    }
  }
  if (!a.parts) return;
  // sums of the walks, one after the other
  float *sums = (float *)marks;  // [walks][lanes V][K], an element's sums side by side
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) sums[((walk * a.lanes + lane) * V + j) * K + k] = dw[k][j];
  __syncthreads();
  const int width = a.lanes * V * K, from = (int)(blockIdx.x % a.passes) * width;
  for (int c = threadIdx.x; c < width; c += kThreads) {
    float v = 0.0f;
    for (int i = 0; i < walks; ++i) v += sums[i * width + c];
    if (from + c < a.dim * K) a.parts[worker * a.dim * K + from + c] = v;
  }
}

// One more row: a lane has the same elements of the state's W - 1 rows and of the new one.
template <class E, int W>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(ConvArgs a, E *state, int64_t slots, const int64_t *slot_of, int64_t first) {
  constexpr int V = kPack<E>;
  const int packs = (a.dim + V - 1) / V;
  const int64_t i = first + (int64_t)blockIdx.x * kThreads + threadIdx.x, r = i / packs;
  if (r >= a.rows) return;
  const int at = (int)(i - r * packs) * V, n = a.dim - at;
  const int64_t slot = slot_of ? slot_of[r] : r;
  float v[V];
  if (slot < 0 || slot >= slots) {
    if (slot >= slots && at == 0) *a.err = 2;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = 0.0f;
  } else {
    float w[W][V], bias[V], e[W][V];
    E *s = state + slot * (W - 1) * a.dim + at;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) load_floats<E, V>(s + (int64_t)k * a.dim, n, e[k]);
    load_floats<E, V>((const E *)a.x + r * a.xs + at, n, e[W - 1]);
    load_weights<W, V>(a, at, w, bias);
    result<W, V>(e, w, bias, v);
    if (a.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= sigmoid(v[j]);
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) store_floats<E, V>(s + (int64_t)k * a.dim, n, e[k + 1]);
  }
  if (a.y) store_floats<E, V>((E *)a.y + r * a.ys + at, n, v);
}

}  // namespace

struct tbe_conv_t : DenseBase {
  int dim, width, dtype;
  bool silu;
  int64_t max_bags, max_rows;
  int32_t *err = nullptr;
  float *parts = nullptr;
};

namespace {

// Lanes of a row (a power of two up to kThreads), and how often so many lanes' elements go into one
void lanes_of(ConvArgs &a, int V, int walk) {
  const int packs = (a.dim + V - 1) / V;
  a.lanes = 1;
  while (a.lanes < packs && a.lanes < kThreads) a.lanes *= 2;
  a.passes = (packs + a.lanes - 1) / a.lanes;
  a.tiles = divide_up(a.rows, (int64_t)kThreads / a.lanes * walk);
}
int64_t tail_groups(const ConvArgs &a, int width, int pack) {  // of lanes behind the tiles, for what is a bag's own
  return divide_up(width > 1 && (a.last || a.dbefore) ? a.bags * (width - 1) * divide_up(a.dim, pack) : a.bags, kThreads);
}

template <class E, int W>
int forward(ConvArgs a, hipStream_t st) {
  lanes_of(a, kPack<E>, kRows);
  const int64_t groups = a.tiles * a.passes + tail_groups(a, W, kPack<E>);
  const size_t lds = (size_t)kThreads / a.lanes * kRows * sizeof(int);
  for (int64_t done = 0; done < groups; done += most_groups(kThreads)) {
    a.first_group = done;
    conv_kernel<E, W><<<dim3((unsigned)std::min(groups - done, most_groups(kThreads))), kThreads, lds, st>>>(a);
  }
  return check_launch();
}

int64_t workers_of(const ConvArgs &a) { return std::max<int64_t>(1, std::min(a.tiles, std::max<int64_t>(kMostParts / a.passes, 64))); }

template <class E, int W>
int backward(ConvArgs a, float *dweight, float *dbias, hipStream_t st) {
  lanes_of(a, kGradPack<E>, grad_rows(W));
  const int64_t workers = workers_of(a), groups = workers * a.passes + tail_groups(a, W, 1);
  const size_t lds = std::max((size_t)(kThreads / a.lanes * grad_rows(W) + W - 1) * sizeof(int), (size_t)kThreads * kGradPack<E> * (W + 1) * sizeof(float));
  for (int64_t done = 0; done < groups; done += most_groups(kThreads)) {  // one launch, unless the earlier rows are of 2^32 elements
    a.first_group = done;
    conv_grad_kernel<E, W><<<dim3((unsigned)std::min(groups - done, most_groups(kThreads))), kThreads, lds, st>>>(a, workers);
  }
  if (a.parts) sum_parts(a.parts, workers, (int64_t)a.dim * (W + 1), W + 1, W, dweight, dbias, nullptr, st);
  return check_launch();
}

template <class E, int W>
int step(ConvArgs a, void *state, int64_t slots, const int64_t *slot_of, hipStream_t st) {
  const int64_t groups = divide_up(a.rows * ((a.dim + kPack<E> - 1) / kPack<E>), kThreads);
  for (int64_t done = 0; done < groups; done += most_groups(kThreads))
    conv_step_kernel<E, W><<<dim3((unsigned)std::min(groups - done, most_groups(kThreads))), kThreads, 0, st>>>(a, (E *)state, slots, slot_of, done * kThreads);
  return check_launch();
}

// call<E, W>() for the handle's type and width
template <class E, class F>
int of_width(int width, F call) {
  switch (width) {
    case 1: return call.template operator()<E, 1>();
    case 2: return call.template operator()<E, 2>();
    case 3: return call.template operator()<E, 3>();
    case 4: return call.template operator()<E, 4>();
    case 5: return call.template operator()<E, 5>();
    case 6: return call.template operator()<E, 6>();
    case 7: return call.template operator()<E, 7>();
    default: return call.template operator()<E, 8>();
  }
}
template <class F>
int of_handle(tbe_conv_handle s, F call) {
  if (s->dtype == TBE_FP32) return of_width<float>(s->width, call);
  if (s->dtype == TBE_FP16) return of_width<_Float16>(s->width, call);
  return of_width<__bf16>(s->width, call);
}

struct Forward {
  ConvArgs a;
  hipStream_t st;
  template <class E, int W> int operator()() const { return forward<E, W>(a, st); }
};
struct Backward {
  ConvArgs a;
  float *dweight, *dbias;
  hipStream_t st;
  template <class E, int W> int operator()() const { return backward<E, W>(a, dweight, dbias, st); }
};
struct Step {
  ConvArgs a;
  void *state;
  int64_t slots;
  const int64_t *slot_of;
  hipStream_t st;
  template <class E, int W> int operator()() const { return step<E, W>(a, state, slots, slot_of, st); }
};

int check_batch(tbe_conv_handle s, const tbe_conv_batch *b, bool bags) {
  if (int rc = check_handle(s)) return rc;
  if (!b) return report(TBE_EINVAL, "null batch");
  if (b->rows < 0 || (bags && b->bags < 0)) return report(TBE_EINVAL, "negative number of bags or rows");
  if (bags && (b->bags > s->max_bags || b->rows > s->max_rows)) return report(TBE_ELIMIT, "more bags or rows than the handle was created for");
  if (!known_dtype(b->weight_dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (bags && b->bags == 0 && b->rows > 0) return report(TBE_EINVAL, "rows without a bag");
  if (bags && b->bags > 0 && !b->d_offsets) return report(TBE_EINVAL, "null offsets");
  if (!b->d_weight || (b->rows > 0 && !b->d_x)) return report(TBE_EINVAL, "null rows or weights");
  if (b->rows > 0 && b->x_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  return TBE_OK;
}
// what a batch's bags share, or have beside their rows
struct Shared {
  Span weight, bias, before, offsets;
  int64_t bag_bytes;
  Shared(tbe_conv_handle s, const tbe_conv_batch *b, bool with_bags = true) {
    const int each = elem_bytes(b->weight_dtype);
    bag_bytes = (with_bags ? b->bags : 0) * (s->width - 1) * s->dim * elem_bytes(s->dtype);
    weight = span(b->d_weight, (int64_t)s->dim * s->width * each), bias = span(b->d_bias, (int64_t)s->dim * each);
    before = of_bags(b->d_before), offsets = with_bags ? span(b->d_offsets, (b->bags + 1) * 8) : Span{};
  }
  Span of_bags(const void *p) const { return span(p, bag_bytes); }
};
ConvArgs args_of(tbe_conv_handle s, const tbe_conv_batch *b) {
  ConvArgs a{};
  a.x = b->d_x, a.xs = b->x_stride, a.weight = b->d_weight, a.bias = b->d_bias, a.weight_dtype = b->weight_dtype;
  a.off = b->d_offsets, a.bags = b->bags, a.rows = b->rows, a.before = s->width > 1 ? b->d_before : nullptr;
  a.dim = s->dim, a.silu = s->silu, a.err = s->err;
  return a;
}

}  // namespace

extern "C" {

int tbe_conv_create(tbe_conv_handle *out, int32_t dim, int32_t width, int32_t dtype, int32_t silu, int64_t max_bags, int64_t max_rows) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (dim < 1 || dim > 65536) return report(TBE_EINVAL, "dim outside 1 .. 65536");
  if (width < 1 || width > kMostWidth) return report(TBE_EINVAL, "width outside 1 .. 8");
  if (!known_dtype(dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (max_bags < 0 || max_rows < 0) return report(TBE_EINVAL, "negative number of bags or rows");
  if (max_bags > (1ll << 38) / dim || max_rows > (1ll << 38) / dim || max_bags >= INT32_MAX)
    return report(TBE_ELIMIT, "more than 2^38 elements, or 2^31 bags");
  tbe_conv_t *s = new (std::nothrow) tbe_conv_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->dim = dim, s->width = width, s->dtype = dtype, s->silu = silu != 0, s->max_bags = max_bags, s->max_rows = max_rows;
  ConvArgs a{};
  a.dim = dim, a.rows = max_rows;
  lanes_of(a, dtype == TBE_FP32 ? kGradPack<float> : kGradPack<_Float16>, grad_rows(width));
  const size_t floats = (size_t)workers_of(a) * dim * (width + 1);
  char *block = nullptr;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&block, 256 + floats * sizeof(float));
  if (e == hipSuccess) e = hipMemset(block, 0, 256);
  if (e != hipSuccess) {
    (void)hipFree(block);
    delete s;
    return report_hip(e);
  }
  s->err = (int32_t *)block;
  s->parts = (float *)(block + 256);
  *out = s;
  return TBE_OK;
}

int tbe_conv_destroy(tbe_conv_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->err);
  delete s;
  return TBE_OK;
}

int tbe_conv_forward(tbe_conv_handle s, const tbe_conv_batch *b, void *d_y, int64_t y_stride, void *d_last, void *stream) {
  if (int rc = check_batch(s, b, true)) return rc;
  if (b->rows > 0 && !d_y) return report(TBE_EINVAL, "null results");
  if (b->rows > 0 && y_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  const Span x = span(b->d_x, s->dim, b->x_stride, b->rows, elem_bytes(s->dtype)), y = span(d_y, s->dim, y_stride, b->rows, elem_bytes(s->dtype));
  const Shared shared(s, b);
  if (int rc = check_apart({y, shared.of_bags(d_last)}, {x, shared.before, shared.weight, shared.bias, shared.offsets})) return rc;
  if (b->bags == 0) return TBE_OK;
  ConvArgs a = args_of(s, b);
  a.y = d_y, a.ys = y_stride, a.last = d_last;
  return of_handle(s, Forward{a, (hipStream_t)stream});
}

int tbe_conv_backward(tbe_conv_handle s, const tbe_conv_batch *b, const void *d_dy, int64_t dy_stride, const void *d_dlast, void *d_dx,
                      int64_t dx_stride, float *d_dweight, float *d_dbias, void *d_dbefore, void *stream) {
  if (int rc = check_batch(s, b, true)) return rc;
  if (b->rows > 0 && (!d_dy || !d_dx)) return report(TBE_EINVAL, "null gradients");
  if (b->rows > 0 && (dy_stride < s->dim || dx_stride < s->dim)) return report(TBE_EINVAL, "a stride below dim");
  const int bytes = elem_bytes(s->dtype);
  const Shared shared(s, b);
  if (int rc = check_apart({span(d_dx, s->dim, dx_stride, b->rows, bytes), shared.of_bags(d_dbefore), span(d_dweight, (int64_t)s->dim * s->width * 4), span(d_dbias, (int64_t)s->dim * 4)},
                           {span(b->d_x, s->dim, b->x_stride, b->rows, bytes), span(d_dy, s->dim, dy_stride, b->rows, bytes), shared.of_bags(d_dlast), shared.before,
                            shared.weight, shared.bias, shared.offsets}))
    return rc;
  if (b->bags == 0 && !d_dweight && !d_dbias) return TBE_OK;
  ConvArgs a = args_of(s, b);
  a.dy = d_dy, a.dys = dy_stride, a.dx = d_dx, a.dxs = dx_stride;
  a.dlast = s->width > 1 ? d_dlast : nullptr, a.dbefore = s->width > 1 ? d_dbefore : nullptr;
  a.parts = d_dweight || d_dbias ? s->parts : nullptr;
  return of_handle(s, Backward{a, d_dweight, d_dbias, (hipStream_t)stream});
}

int tbe_conv_step(tbe_conv_handle s, const tbe_conv_batch *b, void *d_state, int64_t slots, const int64_t *d_slots, void *d_y, int64_t y_stride,
                  void *stream) {
  if (int rc = check_batch(s, b, false)) return rc;
  if (slots < 0) return report(TBE_EINVAL, "negative number of slots");
  if (b->rows > (1ll << 38) / s->dim) return report(TBE_ELIMIT, "more than 2^38 elements");
  if (b->rows == 0) return TBE_OK;
  if (s->width > 1 && !d_state) return report(TBE_EINVAL, "null states");
  if (!d_slots && b->rows > slots) return report(TBE_EINVAL, "more rows than states");
  if (d_y && y_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  const int bytes = elem_bytes(s->dtype);
  const Span x = span(b->d_x, s->dim, b->x_stride, b->rows, bytes), y = span(d_y, s->dim, y_stride, b->rows, bytes);
  const Span state = span(d_state, slots * (s->width - 1) * s->dim * bytes), of_rows = span(d_slots, b->rows * 8);
  const Shared shared(s, b, false);
  if (int rc = check_apart({y, state}, {shared.weight, shared.bias, of_rows})) return rc;
  if (int rc = check_apart({state}, {x, y})) return rc;
  if (!same_span(x, y))  // (a lane reads a row's elements before it writes them)
    if (int rc = check_apart({y}, {x})) return rc;
  ConvArgs a = args_of(s, b);
  a.y = d_y, a.ys = y_stride;
  return of_handle(s, Step{a, d_state, slots, d_slots, (hipStream_t)stream});
}

int tbe_conv_check(tbe_conv_handle s, void *stream) {
  if (int rc = check_handle(s)) return rc;
  return check_errors(s->err, (hipStream_t)stream);
}

}  // extern "C"
