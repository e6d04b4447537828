// Short causal convolution over the rows of every bag: forward, backward, one row for each of many states.
// Contract: include/tbe.h.
//
//   v_t = bias + sum over j < W of w_j e_{t-W+1+j},  e: a bag's earlier rows and its rows;  y = v or silu(v).
//   With g = dy silu'(v):  de_i = sum over k < W of w_{W-1-k} g_{i+k} (rows of the bag),  dw_j = sum over t of g_t e_{t-W+1+j},  dbias = sum of g.
//
// Bound by memory.  A workgroup takes a tile of rows wherever bags begin; a lane walks V elements of kRows rows in a row down, with the
// last W - 1 rows in registers, after up to W - 1 rows in front of its own that it reads once more (from the caches).  Where bags start within the
// tile is written to LDS first.  The backward walks the same way and W - 1 rows on: it finds v again, has the sums of the last W - 1
// rows' gradients in registers and gives a row up when the last result that sees it is done, or where the bag ends.
#include <algorithm>
#include <new>

#include "tbe_rows.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 16;                  // of a lane in a tile
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

template <class E> constexpr int kPack = 16 / sizeof(E) < 8 ? 4 : 8;
constexpr int kGradPack = 4;

// how many of the ascending offsets[0 .. n) are at most `row`, the same in all lanes of a wavefront: 64 places are looked at at once
__device__ inline int64_t count_up_to(const int64_t *off, int64_t n, int64_t row) {
  int64_t lo = 0, hi = n;  // off[i] <= row for i < lo, not for i >= hi
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + (int64_t)(threadIdx.x & 63) * step;
    const uint64_t m = __ballot(at < hi && off[at] <= row);
    const int c = __popcll(m);  // the first c places are
    if (c == 0) return lo;
    lo += (int64_t)(c - 1) * step + 1;
    hi = min(hi, lo + step - 1);
  }
  return lo;
}

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

// The state of a walk: the last W - 1 rows of e (the latest last)
template <int W, int V>
struct Ring {
  float e[W > 1 ? W - 1 : 1][V];
};

template <class E, int W, int V>
__device__ inline void fill_before(Ring<W, V> &ring, const ConvArgs &a, int64_t bag, int at, int n) {
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    if (a.before) load_floats<E, V>((const E *)a.before + (bag * (W - 1) + k) * a.dim + at, n, ring.e[k]);
    else
#pragma unroll
      for (int j = 0; j < V; ++j) ring.e[k][j] = 0.0f;
  }
}

// the rows in front of row r (which does not start a bag, or the ring is filled again): those of its bag, and the earlier ones of that bag
template <class E, int W, int V>
__device__ inline void fill_ring(Ring<W, V> &ring, const ConvArgs &a, const int *marks, int64_t r0, int64_t r, Head head, int at, int n) {
  if constexpr (W > 1) {
    int64_t start = head.start, bag = head.bag;
    int k = 1;
    for (; k < W && r - k >= r0; ++k)
      if (marks[r - k - r0] >= 0) {
        start = r - k, bag = marks[r - k - r0];
        break;
      }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      const int64_t i = r - (W - 1) + k;
      if (i >= start && i >= 0) load_floats<E, V>((const E *)a.x + i * a.xs + at, n, ring.e[k]);
      else if (a.before && i - start + (W - 1) >= 0) load_floats<E, V>((const E *)a.before + (bag * (W - 1) + (i - start + W - 1)) * a.dim + at, n, ring.e[k]);
      else
#pragma unroll
        for (int j = 0; j < V; ++j) ring.e[k][j] = 0.0f;
    }
  }
}

template <int W, int V>
__device__ inline void push(Ring<W, V> &ring, const float (&x)[V]) {
#pragma unroll
  for (int k = 0; k + 1 < W - 1; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) ring.e[k][j] = ring.e[k + 1][j];
  if constexpr (W > 1)
#pragma unroll
    for (int j = 0; j < V; ++j) ring.e[W - 2][j] = x[j];
}

template <int W, int V>
__device__ inline void load_weights(const ConvArgs &a, int at, float (&w)[W][V], float (&bias)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const bool in = at + j < a.dim;
    bias[j] = in && a.bias ? load_param(a.bias, a.weight_dtype, at + j) : 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k][j] = in ? load_param(a.weight, a.weight_dtype, (int64_t)(at + j) * W + k) : 0.0f;
  }
}

template <int W, int V>
__device__ inline void result(const Ring<W, V> &ring, const float (&x)[V], const float (&w)[W][V], const float (&bias)[V], float (&v)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    v[j] = bias[j];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) v[j] += w[k][j] * ring.e[k][j];
    v[j] += w[W - 1][j] * x[j];
  }
}

// Row m of the bag's last W - 1 ones, for the lanes behind the tiles: from the rows or the earlier ones.  GRAD: an empty bag's dbefore, which is its dlast.
template <class E, int W, bool GRAD>
__device__ inline void bag_ends(const ConvArgs &a, int64_t i) {
  if constexpr (W > 1) {
    const int64_t per_bag = (int64_t)(W - 1) * a.dim, b = i / per_bag;
    if (b >= a.bags) return;
    const int64_t s = a.off[b], e = a.off[b + 1];
    const int64_t in = i - b * per_bag;
    if (s > e || s < 0 || e > a.rows || (b == 0 && s != 0) || (b == a.bags - 1 && e != a.rows)) {
      if (in == 0) *a.err = 1;
      return;
    }
    if (GRAD) {
      if (s == e) ((E *)a.dbefore)[i] = a.dlast ? ((const E *)a.dlast)[i] : (E)0.0f;
      return;
    }
    const int m = (int)(in / a.dim), d = (int)(in - (int64_t)m * a.dim);
    const int64_t r = e - (W - 1) + m;
    ((E *)a.last)[i] = r >= s ? ((const E *)a.x)[r * a.xs + d] : a.before ? ((const E *)a.before)[b * per_bag + (r - s + W - 1) * a.dim + d] : (E)0.0f;
  }
}
// the same look at the offsets where there are no such lanes
__device__ inline void look_over(const ConvArgs &a, int64_t b) {
  if (b >= a.bags) return;
  const int64_t s = a.off[b], e = a.off[b + 1];
  if (s > e || s < 0 || e > a.rows || (b == 0 && s != 0) || (b == a.bags - 1 && e != a.rows)) *a.err = 1;
}

template <class E, int W>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvArgs a) {
  constexpr int V = kPack<E>;
  extern __shared__ int marks[];
  const int64_t group = a.first_group + blockIdx.x;
  if (group >= a.tiles * a.passes) {
    const int64_t i = (group - a.tiles * a.passes) * kThreads + threadIdx.x;
    if (W > 1 && a.last) bag_ends<E, W, false>(a, i);
    else look_over(a, i);
    return;
  }
  const int64_t tile = group / a.passes;
  const int walks = kThreads / a.lanes, tile_rows = walks * kRows;
  const int64_t r0 = tile * tile_rows, r1 = min(r0 + tile_rows, a.rows);
  const Head head = mark_tile(a, r0, r1, marks, tile_rows);
  const int at = ((int)(group % a.passes) * a.lanes + (threadIdx.x & (a.lanes - 1))) * V, n = a.dim - at;
  const int64_t first = r0 + threadIdx.x / a.lanes * kRows;
  if (n <= 0 || first >= r1) return;
  float w[W][V], bias[V];
  load_weights<W, V>(a, at, w, bias);
  Ring<W, V> ring;
  fill_ring<E, W, V>(ring, a, marks, r0, first, head, at, n);
  const int64_t end = min(first + kRows, r1);
#pragma unroll 4
  for (int64_t r = first; r < end; ++r) {
    float x[V], v[V];
    load_floats<E, V>((const E *)a.x + r * a.xs + at, n, x);
    const int b = marks[r - r0];
    if (b >= 0) fill_before<E, W, V>(ring, a, b, at, n);
    result<W, V>(ring, x, w, bias, v);
    if (a.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= sigmoid(v[j]);
    }
    store_floats<E, V>((E *)a.y + r * a.ys + at, n, v);
    push<W, V>(ring, x);
  }
}

template <class E, int W>
__global__ __launch_bounds__(kThreads) void conv_grad_kernel(ConvArgs a, int64_t workers) {
  constexpr int V = kGradPack, K = W + 1;  // sums of an element: W of dw, one of dbias
  extern __shared__ int marks[];           // tile_rows + W - 1 of them, and then the sums of the walks
  if ((int64_t)blockIdx.x >= workers * a.passes) {
    const int64_t i = ((int64_t)blockIdx.x - workers * a.passes) * kThreads + threadIdx.x;
    if (W > 1 && a.dbefore) bag_ends<E, W, true>(a, i);
    else look_over(a, i);
    return;
  }
  const int lane = threadIdx.x & (a.lanes - 1), walk = threadIdx.x / a.lanes, walks = kThreads / a.lanes, tile_rows = walks * kRows;
  const int64_t worker = blockIdx.x / a.passes;
  const int at = ((int)(blockIdx.x % a.passes) * a.lanes + lane) * V, n = a.dim - at;
  float w[W][V], bias[V], dw[K][V];
  if (n > 0) load_weights<W, V>(a, at, w, bias);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[k][j] = 0.0f;
  for (int64_t tile = worker; tile < a.tiles; tile += workers) {
    const int64_t r0 = tile * tile_rows, r1 = min(r0 + tile_rows, a.rows);
    __syncthreads();  // the marks of the tile before
    const Head head = mark_tile(a, r0, min(r1 + W - 1, a.rows), marks, tile_rows + W - 1);
    const int64_t first = r0 + walk * kRows, end = min(first + kRows, r1);
    if (n <= 0 || first >= r1) continue;
    Ring<W, V> ring;
    fill_ring<E, W, V>(ring, a, marks, r0, first, head, at, n);
    float acc[W][V];  // acc[k]: what rows r - k have had so far
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[k][j] = 0.0f;
    int64_t bag = -1, start = -1;  // of the bag that started within these rows
    // Row p has all of its gradient, d.  `ends`: the bag, `of`, ends in front of row e, so its last rows have a part of dlast.
    auto give = [&](int64_t p, const float(&d)[V], bool ends, int64_t e, int64_t of) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = d[j];
      if (ends && a.dlast && p >= e - (W - 1)) {
        float t[V];
        load_floats<E, V>((const E *)a.dlast + (of * (W - 1) + (p - e + W - 1)) * a.dim + at, n, t);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] += t[j];
      }
      if (start >= 0 && p < start) {  // an earlier row of a bag that starts here
        if (a.dbefore && p >= start - (W - 1)) store_floats<E, V>((E *)a.dbefore + (of * (W - 1) + (p - start + W - 1)) * a.dim + at, n, o);
      } else if (p >= first && p < end) {
        store_floats<E, V>((E *)a.dx + p * a.dxs + at, n, o);
      }
    };
    auto finish = [&](int64_t e) {  // the bag ends in front of row e: its rows e - 1 .. e - W + 1 (and earlier ones) are done
      int64_t of = bag >= 0 ? bag : head.bag;
      if (bag < 0 && a.dlast)  // it started in front of these rows, in this tile or before
        for (int64_t q = first - 1; q >= r0; --q)
          if (marks[q - r0] >= 0) {
            of = marks[q - r0];
            break;
          }
#pragma unroll
      for (int k = W - 1; k >= 1; --k) give(e - k, acc[k], true, e, of);
    };
    const int64_t stop = min(end + W - 1, a.rows);
    int64_t r = first;
    bool open = false;  // rows of `first` and after have something in acc
    for (; r < stop; ++r) {
      const int b = marks[r - r0];
      // acc[k] belongs to row r - k from here on
#pragma unroll
      for (int k = W - 1; k >= 1; --k)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] = acc[k - 1][j];
#pragma unroll
      for (int j = 0; j < V; ++j) acc[0][j] = 0.0f;
      if (b >= 0) {
        if (open) finish(r);
        if (r >= end) {  // the next walk's
          open = false;
          break;
        }
        fill_before<E, W, V>(ring, a, b, at, n);
        bag = b, start = r;
#pragma unroll
        for (int k = 1; k < W; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) acc[k][j] = 0.0f;
      }
      open = true;
      float x[V], g[V], v[V];
      load_floats<E, V>((const E *)a.x + r * a.xs + at, n, x);
      load_floats<E, V>((const E *)a.dy + r * a.dys + at, n, g);
      if (a.silu) {
        result<W, V>(ring, x, w, bias, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float f = sigmoid(v[j]);
          g[j] *= f * (1.0f + v[j] * (1.0f - f));
        }
      }
      if (r < end) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
#pragma unroll
          for (int k = 0; k < W - 1; ++k) dw[k][j] += g[j] * ring.e[k][j];
          dw[W - 1][j] += g[j] * x[j];
          dw[W][j] += g[j];
        }
      }
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] += w[W - 1 - k][j] * g[j];
      give(r - (W - 1), acc[W - 1], false, 0, bag);
      push<W, V>(ring, x);
    }
    // Rows of the walk that are still open: the data end, so does their bag.  (Otherwise the walk has gone W - 1 rows on and given up all of its own.)
    if (open && r == a.rows) {
#pragma unroll
      for (int k = W - 1; k >= 1; --k)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[k][j] = acc[k - 1][j];
      finish(r);
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
    float w[W][V], bias[V], x[V];
    Ring<W, V> ring;
    E *s = state + slot * (W - 1) * a.dim + at;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) load_floats<E, V>(s + (int64_t)k * a.dim, n, ring.e[k]);
    load_floats<E, V>((const E *)a.x + r * a.xs + at, n, x);
    load_weights<W, V>(a, at, w, bias);
    result<W, V>(ring, x, w, bias, v);
    if (a.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= sigmoid(v[j]);
    }
    push<W, V>(ring, x);
#pragma unroll
    for (int k = 0; k < W - 1; ++k) store_floats<E, V>(s + (int64_t)k * a.dim, n, ring.e[k]);
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
void lanes_of(ConvArgs &a, int V) {
  const int packs = (a.dim + V - 1) / V;
  a.lanes = 1;
  while (a.lanes < packs && a.lanes < kThreads) a.lanes *= 2;
  a.passes = (packs + a.lanes - 1) / a.lanes;
  a.tiles = divide_up(a.rows, (int64_t)kThreads / a.lanes * kRows);
}
int64_t tail_groups(const ConvArgs &a, int width) {  // of lanes behind the tiles, for what is a bag's own
  return divide_up(width > 1 && (a.last || a.dbefore) ? a.bags * (width - 1) * a.dim : a.bags, kThreads);
}

template <class E, int W>
int forward(ConvArgs a, hipStream_t st) {
  lanes_of(a, kPack<E>);
  const int64_t groups = a.tiles * a.passes + tail_groups(a, W);
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
  lanes_of(a, kGradPack);
  const int64_t workers = workers_of(a), groups = workers * a.passes + tail_groups(a, W);
  if (groups > most_groups(kThreads)) return report(TBE_ELIMIT, "more bags than one launch can take");
  const size_t lds = std::max((size_t)(kThreads / a.lanes * kRows + W - 1) * sizeof(int), (size_t)kThreads * kGradPack * (W + 1) * sizeof(float));
  conv_grad_kernel<E, W><<<dim3((unsigned)groups), kThreads, lds, st>>>(a, workers);
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
  lanes_of(a, kGradPack);
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
  if (b->rows > 0 && d_y == b->d_x) return report(TBE_EINVAL, "the output is one of the inputs");
  if (d_last && d_last == b->d_before) return report(TBE_EINVAL, "the output is one of the inputs");
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
  if (b->rows > 0 && (d_dx == b->d_x || d_dx == d_dy)) return report(TBE_EINVAL, "an output is one of the inputs");
  if (d_dbefore && (d_dbefore == b->d_before || d_dbefore == d_dlast)) return report(TBE_EINVAL, "an output is one of the inputs");
  if (d_dbias && !d_dweight) return report(TBE_EINVAL, "the gradient of the bias comes with that of the weights");
  if (b->bags == 0 && !d_dweight) return TBE_OK;
  ConvArgs a = args_of(s, b);
  a.dy = d_dy, a.dys = dy_stride, a.dx = d_dx, a.dxs = dx_stride;
  a.dlast = s->width > 1 ? d_dlast : nullptr, a.dbefore = s->width > 1 ? d_dbefore : nullptr;
  a.parts = d_dweight ? s->parts : nullptr;
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
  ConvArgs a = args_of(s, b);
  a.y = d_y, a.ys = y_stride;
  return of_handle(s, Step{a, d_state, slots, d_slots, (hipStream_t)stream});
}

int tbe_conv_check(tbe_conv_handle s, void *stream) {
  if (int rc = check_handle(s)) return rc;
  return check_errors(s->err, (hipStream_t)stream);
}

}  // extern "C"
