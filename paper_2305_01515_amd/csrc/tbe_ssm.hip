// Selective scan over the rows of every bag: forward, backward, one row for each of many states.
// Contract: include/tbe.h.
//
//   D_t = log(1 + exp(delta_t + bias)),  h_t[n] = exp(D_t a[n]) h_{t-1}[n] + D_t b_t[n] x_t,  y_t = (sum_n c_t[n] h_t[n] + skip x_t) silu(z_t).
//   Backward, with dv = dy silu(z):  g_t = c_t dv_t + exp(D_{t+1} a) g_{t+1} (a bag's last row: + dlast),  w_t = exp(D_t a) h_{t-1},
//   dx = skip dv + D sum_n g b,  dD = sum_n g w a + x sum_n g b,  da = sum_t g w D,  db = sum over elements of g D x,  dc = sum of dv h.
//
// Bound by vector instructions: an element and a state take an exponential (two turns of the vector unit) and four more, 16 states 96 turns, for 8 to
// 14 bytes of rows in 16 bits.  So the rows are gone through once where that can be, and no lane idles:
//   units    The rows are cut every `unit` rows.  A bag of up to two units is not cut: the unit it starts in goes on to its end.
//   ends     Units whose end cuts a bag find the state there from a zero one (or the bag's start), and the sum of the D: the
//            product of the decays is the exponential of a times that                          (ssm_ends_kernel)
//   join     states at the cuts, by a scan over the units in segments and one over the segments (ssm_join_kernel, ssm_segments_kernel)
//   rows     every unit from the state before it                                                (ssm_kernel, ssm_grad_kernel)
// Where no bag is longer than two units, `ends` and `join` find nothing to do.
// Forward: a lane has an element with all of its states in registers, b and c come from LDS.  Backward: a lane has four states of an
// element, so that 8 rows' w and decays stay in registers on the way back; states before every 8th row were saved by the forward.
// 245760 rows of 128 in bags of 30, bfloat16, 16 states, gated: forward 200 us (0.86 of it vector instructions), backward 880 us (0.6 of it); three bags of 100 k
// rows of 64 in fp32: forward 125 us and 86 for the ends, backward 510 and 91, joins 34 + 17 us each way.
// Other numbers of states, the same short bags: 4 and 8 take what 16 do or a little more; 24 of them 370 us forward, 1533 back, 64 of them 780 and 3385.
#include <algorithm>
#include <new>
#include <type_traits>

#include "tbe_rows.h"

using namespace tbe;

namespace {

constexpr int kSaved = 8;        // states before every so many rows are what the backward goes from: that many rows' w and decays fit its registers
constexpr int kSegment = 64;     // units that a lane of `join` goes through
constexpr int kMostStates = 64;
constexpr int kThreads = 256;
constexpr int kGradWaves = 2048;    // wavefronts of the backward, as many as the GPU holds at once

struct Unit {
  int64_t begin;  // first row
  int32_t bag;    // that its first row by count belongs to
  int32_t cut;    // 1: begins within a bag
};

struct SsmArgs {
  const void *x, *delta, *z, *b, *c, *dy;
  int64_t xs, ts, zs, bs, cs, dys;
  const float *a, *skip, *bias, *h0, *dlast;
  const int64_t *off;
  int64_t bags, rows, h0s;
  int dim, states, groups;
  void *y, *dx, *ddelta, *dz, *db, *dc;
  int64_t ys;
  float *last, *saved, *dh0;
  // scratch
  Unit *units;
  int2 *marks;      // [rows]: the bag that starts at a row, the bag whose last row it is (-1: none)
  float *ends;      // [units][dim][NP]: states at the ends; `join` puts what is before (behind) each unit in their place
  float *spans;     // [units][dim]: sums of D
  float *reach;     // [units][dim]: sum of D from the segment's start; negative: nothing of it gets here
  float *seg_state; // [segments][dim][NP]
  float *seg_reach; // [segments][dim]
  float *seg_start; // [segments][dim][NP]
  int32_t *seg_says; // [segments]: whether a unit of it says anything
  float *parts, *shared;
  int32_t *err;
  int64_t count;    // units
  int unit;         // rows of one
  int waves;        // of 64 elements that a row has
  int64_t workers;
  int blocks;       // workgroups that a row has in the backward
};

// The units and the marks of their rows, what empty bags have; offsets that do not ascend from 0 to rows are reported.
// empty_to (or null): [bags, dim, states] that an empty bag has of empty_from (null: zero).
constexpr int kMostUnit = 128;
__global__ __launch_bounds__(kThreads) void ssm_prepare_kernel(SsmArgs a, int64_t bag_groups, float *empty_to, const float *empty_from, int64_t empty_stride) {
  __shared__ int2 marks[kThreads / 64][kMostUnit];
  const int lane = threadIdx.x & 63;
  if (blockIdx.x < bag_groups) {
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    bool empty = false;
    if (b < a.bags) {
      const int64_t s = a.off[b], e = a.off[b + 1];
      if (s > e || s < 0 || e > a.rows || (b == 0 && s != 0) || (b == a.bags - 1 && e != a.rows)) *a.err = 1;
      else empty = s == e;
    }
    if (!empty_to) return;
    const int64_t n = (int64_t)a.dim * a.states;
    for (uint64_t m = __ballot(empty); m; m &= m - 1) {
      const int64_t of = b - lane + __builtin_ctzll(m);
      for (int64_t i = lane; i < n; i += 64) empty_to[of * n + i] = empty_from ? empty_from[of * empty_stride + i] : 0.0f;
    }
    return;
  }
  const int64_t k = ((int64_t)blockIdx.x - bag_groups) * (kThreads / 64) + threadIdx.x / 64;
  const int64_t r = k * a.unit, to = min(r + a.unit, a.rows);
  const bool some = k < a.count;  // a wavefront without a unit waits with the others
  Unit u{a.rows, 0, 0};
  int2 *m = marks[threadIdx.x / 64];
  int64_t head = 0;
  if (some) {
    head = max(count_up_to(a.off, a.bags, r) - 1, (int64_t)0);
    const int64_t s = a.off[head], e = a.off[head + 1];
    u.bag = (int)head;
    u.cut = s != r && e - s > 2 * a.unit;
    // (offsets that do not ascend: the unit still begins within its own rows and those of the next two)
    u.begin = s == r || u.cut ? r : min(max(e, r), min(r + 2 * a.unit, a.rows));
    for (int i = lane; i < a.unit; i += 64) m[i] = {-1, -1};
  }
  if (lane == 0 && k <= a.count) a.units[k] = u;
  __syncthreads();
  if (some) {
    for (int64_t b = head + lane; b < a.bags; b += 64) {
      const int64_t s = a.off[b], e = a.off[b + 1];
      if (s >= to) break;
      if (e <= s) continue;
      if (s >= r) m[s - r].x = (int)b;
      if (e > r && e <= to) m[e - 1 - r].y = (int)b;
    }
  }
  __syncthreads();
  if (some)
    for (int64_t i = lane; i < to - r; i += 64) a.marks[r + i] = m[i];
}

// D = log(1 + exp(u)): with e = exp(-|u|) and w = 1 + e rounded, log(1 + e) is log(w) and what the rounding left out
__device__ inline float soft(float u) {
  const float e = __builtin_amdgcn_exp2f(fabsf(u) * -kLog2e), w = 1.0f + e;
  return fmaxf(u, 0.0f) + (__builtin_amdgcn_logf(w) * kLn2 + (e - (w - 1.0f)));
}
// a decay's product with a state that may be zero beside an infinite one
__device__ inline float carried(float a2, float span, float h) { return h == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(a2 * span) * h; }

// States n .. n + COUNT - 1 of element d before unit k, as `join` left them
template <int NP, int COUNT>
__device__ inline void start_of(const SsmArgs &a, int64_t k, int d, int n, const float *a2, float (&to)[COUNT]) {
  const float r = a.reach[k * a.dim + d], *h = a.ends + (k * a.dim + d) * NP + n;
  float far[COUNT];
#pragma unroll
  for (int j = 0; j < COUNT; ++j) to[j] = h[j];
  const float *p = a.seg_start + (k / kSegment * a.dim + d) * NP + n;  // (of no meaning where nothing of the segment before gets here)
#pragma unroll
  for (int j = 0; j < COUNT; ++j) far[j] = p[j];
#pragma unroll
  for (int j = 0; j < COUNT; ++j) to[j] += r < 0.0f ? 0.0f : carried(a2[j], r, far[j]);
}

// Waits for loaded numbers here.  Behind a branch that loads, the compiler would wait where they are used first, on the way that has loaded nothing
// too, and for all loads and stores under way: a store's time for each row.
template <int COUNT>
__device__ inline void settle(float (&v)[COUNT]) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) asm volatile("" : "+v"(v[i]));
}

// The lane's number, found again: what follows from it would be kept from block to block in registers that there are not.
__device__ inline int lane_again() {
  int me = threadIdx.x;
  asm volatile("" : "+v"(me));
  return me;
}

// Elements at .. at + V - 1 of a row, those beyond its end being other ones of it.  All lanes go one way, and no v_readlane stands where lanes are masked off:
// a register that has been kept elsewhere comes back in the active lanes only, and what is then read of another lane is something else.
template <class E, int V>
__device__ inline void load_pack_of(const E *row, int dim, int at, Words<E, V> &to) {
  if (dim % V == 0) {
    __builtin_memcpy(to.w, row + min(at, dim - V), sizeof to.w);
  } else {
#pragma unroll
    for (unsigned i = 0; i < sizeof to.w / 4; ++i) {
      if constexpr (sizeof(E) == 4) {
        to.w[i] = ((const uint32_t *)row)[min(at + (int)i, dim - 1)];
      } else {
        const uint16_t *p = (const uint16_t *)row;
        to.w[i] = p[min(at + 2 * (int)i, dim - 1)] | (uint32_t)p[min(at + 2 * (int)i + 1, dim - 1)] << 16;
      }
    }
  }
}

// A wavefront goes down a unit's rows in tiles of 2 V rows of 64 elements: x, delta and z are read in packs of 16 bytes a tile ahead, b, c
// and marks too, and lie in LDS while the tile is gone through.
template <class E, int NP, bool FULL>
__global__ __launch_bounds__(64, NP == 16 && FULL ? 3 : 1) void ssm_kernel(SsmArgs a) {
  constexpr int V = 16 / sizeof(E), T = 2 * V, PACKS = 64 / V;
  __shared__ float bc[T][2 * NP];
  __shared__ Words<E, V> tile[3][T][PACKS];
  const int64_t k = blockIdx.x / a.waves;
  const int wave = (int)(blockIdx.x % a.waves), lane = threadIdx.x;
  const Unit u = a.units[k];
  const int64_t begin = u.begin, end = a.units[k + 1].begin;
  if (begin >= end) return;
  // Lanes beyond the row's end do what the last element's lane does, and write what it writes.
  const int column = min(lane, a.dim - 1 - wave * 64), dc = wave * 64 + column;
  const int group = a.groups > 1 ? wave * 64 / (a.dim / a.groups) : 0, N = a.states;
  const bool gated = a.z;
  Words<E, V> raw[3][2];
  constexpr int PIECES = T * 2 * NP / 64;  // of a tile's b and c
  constexpr int ROWS = 64 / (2 * NP) > 0 ? 64 / (2 * NP) : 1, PARTS = 2 * NP > 64 ? 2 * NP / 64 : 1;
  E shared[PIECES];
  int2 mark;
  auto fetch = [&](int64_t row0) {
    const int me = lane_again(), pack = wave * 64 + me % PACKS * V;  // of a row, that this lane brings
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = min(max(row0 + i * V + me / PACKS, begin), end - 1);
      load_pack_of<E, V>((const E *)a.x + r * a.xs, a.dim, pack, raw[0][i]);
      load_pack_of<E, V>((const E *)a.delta + r * a.ts, a.dim, pack, raw[1][i]);
      if (gated) load_pack_of<E, V>((const E *)a.z + r * a.zs, a.dim, pack, raw[2][i]);
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int n = PARTS > 1 ? p % PARTS * 64 + me : me % (2 * NP), t = PARTS > 1 ? p / PARTS : p * ROWS + me / (2 * NP);
      const int64_t r = min(max(row0 + t, begin), end - 1);
      const int at = group * N + min(n % NP, N - 1);
      shared[p] = n < NP ? ((const E *)a.b)[r * a.bs + at] : ((const E *)a.c)[r * a.cs + at];
    }
    mark = a.marks[min(max(row0 + (lane & (T - 1)), begin), end - 1)];
  };
  const int64_t from = begin & ~(int64_t)(T - 1);
  fetch(from);
  float h[NP], a2[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    a2[n] = FULL || n < N ? a.a[(int64_t)dc * N + n] * kLog2e : 0.0f;
    h[n] = 0.0f;
  }
  if (u.cut) {
    start_of<NP>(a, k, dc, 0, a2, h);
    settle(h);
  }
  const float bias = a.bias ? a.bias[dc] : 0.0f, skip = a.skip ? a.skip[dc] : 0.0f;
  for (int64_t row0 = from; row0 < end; row0 += T) {
    const int lo = (int)max(begin - row0, (int64_t)0), hi = (int)min(end - row0, (int64_t)T);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < 2 || gated) tile[j][i * V + lane / PACKS][lane % PACKS] = raw[j][i];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int n = PARTS > 1 ? p % PARTS * 64 + lane : lane % (2 * NP), t = PARTS > 1 ? p / PARTS : p * ROWS + lane / (2 * NP);
      bc[t][n] = FULL || n % NP < N ? (float)shared[p] : 0.0f;
    }
    const int2 bag_of = mark;
    const bool mine = lane >= lo && lane < hi;
    const uint32_t starts = (uint32_t)__ballot(mine && mark.x >= 0), ends = (uint32_t)__ballot(mine && mark.y >= 0);
    if (row0 + T < end) fetch(row0 + T);
    __syncthreads();
    const E *xt = (const E *)tile[0] + column, *ut = (const E *)tile[1] + column, *zt = (const E *)tile[2] + column;
    E *y = (E *)a.y + (row0 + lo) * a.ys + dc;
    auto put = [&](int t) {  // the state before row t, for the backward
      if (a.saved && (t & (kSaved - 1)) == 0) {
        float *to = a.saved + ((row0 + t) / kSaved * a.dim + dc) * NP;
#pragma unroll
        for (int n = 0; n < NP; n += 4) *(float4 *)(to + n) = make_float4(h[n], h[n + 1], h[n + 2], h[n + 3]);
      }
    };
    auto go = [&](int t, E xe, E ue, E ze) {
      const float xv = (float)xe, step = soft((float)ue + bias), sx = step * xv;
      float v = skip * xv, v2 = 0.0f;
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const float g = __builtin_amdgcn_exp2f(step * a2[n]) * h[n] + sx * bc[t][n];
        h[n] = FULL || n < N ? g : 0.0f;
        (n & 1 ? v2 : v) += bc[t][NP + n] * h[n];
      }
      v += v2;
      if (gated) {
        const float zv = (float)ze;
        v *= zv * sigmoid(zv);
      }
      return v;
    };
    for (int t = lo; t < hi;) {
      constexpr int R = sizeof(E) == 2 ? 2 : 4;
      if (t + R <= hi && (t & (R - 1)) == 0 && !((starts | ends) >> t & ((1 << R) - 1))) {  // without branches between the rows
        put(t);
        float v[R];
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = go(t + i, xt[(t + i) * 64], ut[(t + i) * 64], zt[(t + i) * 64]);
#pragma unroll
        for (int i = 0; i < R; ++i) y[i * a.ys] = (E)v[i];
        y += R * a.ys;
        t += R;
        continue;
      }
      const E xe = xt[t * 64], ue = ut[t * 64], ze = zt[t * 64];
      if (starts >> t & 1) {
        const int64_t bag = __builtin_amdgcn_readlane(bag_of.x, t);
        if (a.h0) {
          const float *p = a.h0 + bag * a.h0s + (int64_t)dc * N;
#pragma unroll
          for (int n = 0; n < NP; n += 4) {
            float v[4];
            load_floats<float, 4>(p + n, FULL ? 4 : N - n, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) h[n + j] = v[j];
          }
          settle(h);
        } else {
#pragma unroll
          for (int n = 0; n < NP; ++n) h[n] = 0.0f;
        }
      }
      put(t);
      const float v = go(t, xe, ue, ze);
      *y = (E)v;
      y += a.ys;
      if ((ends >> t & 1) && a.last) {
        const int64_t bag = __builtin_amdgcn_readlane(bag_of.y, t);
        float *to = a.last + (bag * a.dim + dc) * N;
#pragma unroll
        for (int n = 0; n < NP; n += 4) {
          const float v[4] = {h[n], h[n + 1], h[n + 2], h[n + 3]};
          store_floats<float, 4>(to + n, FULL ? 4 : N - n, v);
        }
      }
      ++t;
    }
  }
}

// gradient of v = sum c h + skip x, from that of y
__device__ inline float before_gate(float dy, bool gated, float z) { return gated ? dy * z * sigmoid(z) : dy; }

// What a unit says.  Forward, one whose end is within a bag: the state there, from zero (the bag began before) or from the bag's start.  BACK, one that begins
// within a bag: exp(D a) g of its first row, from the bag's end or from zero.  Rows are read in tiles as in ssm_kernel.
template <class E, int NP, bool BACK>
__global__ __launch_bounds__(64) void ssm_ends_kernel(SsmArgs a) {
  constexpr int V = 16 / sizeof(E), T = 2 * V, PACKS = 64 / V, R = sizeof(E) == 2 ? 2 : 4;
  __shared__ float bc[T][NP];  // b, or c
  __shared__ Words<E, V> tile[3][T][PACKS];
  const int64_t k = blockIdx.x / a.waves;
  const Unit u = a.units[k], next = a.units[k + 1];
  if (!(BACK ? u.cut : next.cut)) return;
  const bool whole = u.cut && next.cut && u.bag == next.bag, gated = BACK && a.z;
  const int64_t begin = BACK ? u.begin : max(u.begin, a.off[next.bag]);
  const int64_t end = BACK && !whole ? min(next.begin, max(a.off[u.bag + 1], begin)) : next.begin;
  const int wave = (int)(blockIdx.x % a.waves), lane = threadIdx.x, N = a.states;
  const int column = min(lane, a.dim - 1 - wave * 64), dc = wave * 64 + column, group = a.groups > 1 ? wave * 64 / (a.dim / a.groups) : 0;
  Words<E, V> raw[3][2];
  constexpr int NUMBERS = T * NP / 64;
  E shared[NUMBERS];
  auto fetch = [&](int64_t row0) {
    const int me = lane_again(), pack = wave * 64 + me % PACKS * V;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = min(max(row0 + i * V + me / PACKS, begin), end - 1);
      load_pack_of<E, V>(BACK ? (const E *)a.dy + r * a.dys : (const E *)a.x + r * a.xs, a.dim, pack, raw[0][i]);
      load_pack_of<E, V>((const E *)a.delta + r * a.ts, a.dim, pack, raw[1][i]);
      if (gated) load_pack_of<E, V>((const E *)a.z + r * a.zs, a.dim, pack, raw[2][i]);
    }
#pragma unroll
    for (int i = 0; i < NUMBERS; ++i) {
      const int n = me + i * 64;
      const int64_t r = min(max(row0 + n / NP, begin), end - 1);
      const E *from = BACK ? (const E *)a.c + r * a.cs : (const E *)a.b + r * a.bs;
      shared[i] = from[group * N + min(n % NP, N - 1)];
    }
  };
  const int64_t first = (BACK ? end - 1 : begin) & ~(int64_t)(T - 1);
  if (begin < end) fetch(first);
  float h[NP], a2[NP], span = 0.0f;  // BACK, h: what the row before the last one seen gets
  const float *from = BACK ? a.dlast : a.h0;
  const int64_t at = BACK ? (int64_t)u.bag * a.dim * N : next.bag * a.h0s;
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    a2[n] = n < N ? a.a[(int64_t)dc * N + n] * kLog2e : 0.0f;
    h[n] = !whole && from && n < N ? from[at + (int64_t)dc * N + n] : 0.0f;
  }
  const float bias = a.bias ? a.bias[dc] : 0.0f;
  for (int64_t row0 = first; BACK ? row0 + T > begin : row0 < end; row0 += BACK ? -T : T) {
    const int lo = (int)max(begin - row0, (int64_t)0), hi = (int)min(end - row0, (int64_t)T);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < 2 || gated) tile[j][i * V + lane / PACKS][lane % PACKS] = raw[j][i];
#pragma unroll
    for (int i = 0; i < NUMBERS; ++i) (&bc[0][0])[lane + i * 64] = (lane + i * 64) % NP < N ? (float)shared[i] : 0.0f;
    if (BACK ? row0 > begin : row0 + T < end) fetch(row0 + (BACK ? -T : T));
    __syncthreads();
    const E *xt = (const E *)tile[0] + column, *ut = (const E *)tile[1] + column, *zt = (const E *)tile[2] + column;
    auto go = [&](int t) {
      const float step = soft((float)ut[t * 64] + bias), x = (float)xt[t * 64];
      const float s = BACK ? before_gate(x, gated, gated ? (float)zt[t * 64] : 0.0f) : step * x;
      span += step;
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const float decay = __builtin_amdgcn_exp2f(step * a2[n]);
        h[n] = BACK ? decay * (bc[t][n] * s + h[n]) : decay * h[n] + s * bc[t][n];
      }
    };
    for (int n = 0; n < hi - lo;) {  // rows done
      const int t = BACK ? hi - 1 - n : lo + n;
      if (n + R <= hi - lo) {
#pragma unroll
        for (int i = 0; i < R; ++i) go(BACK ? t - i : t + i);
        n += R;
      } else {
        go(t);
        ++n;
      }
    }
  }
  float *to = a.ends + (k * a.dim + dc) * NP;
#pragma unroll
  for (int n = 0; n < NP; n += 4) *(float4 *)(to + n) = make_float4(h[n], h[n + 1], h[n + 2], h[n + 3]);
  a.spans[k * a.dim + dc] = span;
}

// Whether unit k says something to the next one (BACK: the one before), and whether that has a part of what it has heard itself
template <bool BACK>
__device__ inline int says(const SsmArgs &a, int64_t k) {
  const Unit u = a.units[k], next = a.units[k + 1];
  return (BACK ? u.cut : next.cut) ? 1 + (u.cut && next.cut && u.bag == next.bag) : 0;
}

// A segment of units, a lane for each state of each element: what comes before (BACK: behind) each unit, but for what comes before the segment
template <int NP, bool BACK>
__global__ __launch_bounds__(kThreads) void ssm_join_kernel(SsmArgs a, int64_t segments, int groups) {
  const int64_t seg = blockIdx.x / groups, i = (int64_t)(blockIdx.x % groups) * kThreads + threadIdx.x;
  const int64_t k0 = seg * kSegment, k1 = min(k0 + kSegment, a.count);
  const int lane = threadIdx.x & 63;
  // of every unit of the segment, by the lanes of a wavefront
  const int mine = k0 + lane < k1 ? says<BACK>(a, k0 + lane) : 0;
  const uint64_t speak = __ballot(mine > 0), pass = __ballot(mine > 1);
  const int64_t n_all = (int64_t)a.dim * NP;
  const bool in = i < n_all;
  const int64_t ic = in ? i : n_all - 1;
  const int d = (int)(ic / NP), n = (int)(ic % NP);
  if (blockIdx.x % groups == 0 && threadIdx.x == 0) a.seg_says[seg] = speak != 0;
  if (!speak) {  // no cut bag: nothing to be written but that nothing gets through
    if (in && n == 0) a.seg_reach[seg * a.dim + d] = -1.0f;
    if (in) a.seg_state[seg * n_all + i] = 0.0f;
    // the first unit (BACK: the last) may be told something by the segment before
    const int64_t k = BACK ? k1 - 1 : k0;
    if (in) a.ends[k * n_all + i] = 0.0f;
    if (in && n == 0) a.reach[k * a.dim + d] = 0.0f;
    return;
  }
  const float a2 = n < a.states ? a.a[(int64_t)d * a.states + n] * kLog2e : 0.0f;
  float st = 0.0f, sum = 0.0f;  // sum < 0: nothing of what comes before the segment gets here
  constexpr int R = 16;  // loads under way
  for (int64_t j0 = 0; j0 < k1 - k0; j0 += R) {
    float e[R], s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t j = j0 + r, k = BACK ? k1 - 1 - j : k0 + j;
      const bool some = j < k1 - k0 && (speak >> (k - k0) & 1);
      e[r] = some ? a.ends[k * n_all + ic] : 0.0f;
      s[r] = some ? a.spans[k * a.dim + d] : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t j = j0 + r, k = BACK ? k1 - 1 - j : k0 + j;
      if (j >= k1 - k0) continue;
      if (in) a.ends[k * n_all + i] = st;
      if (in && n == 0) a.reach[k * a.dim + d] = sum;
      const int64_t bit = k - k0;
      if (pass >> bit & 1) {
        st = carried(a2, s[r], st) + e[r];
        sum = sum < 0.0f ? sum : sum + s[r];
      } else {
        st = e[r];  // zero where it says nothing
        sum = -1.0f;
      }
    }
  }
  if (!in) return;
  a.seg_state[seg * n_all + i] = st;
  if (n == 0) a.seg_reach[seg * a.dim + d] = sum;
}

// What comes before (BACK: behind) each segment
template <int NP, bool BACK>
__global__ __launch_bounds__(64) void ssm_segments_kernel(SsmArgs a, int64_t segments) {
  const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x, n_all = (int64_t)a.dim * NP;
  bool any = false;  // else nobody asks
  for (int64_t k = threadIdx.x; k < segments; k += 64) any = any || a.seg_says[k] != 0;
  if (!__any(any) || i >= n_all) return;
  const int d = (int)(i / NP), n = (int)(i % NP);
  const float a2 = n < a.states ? a.a[(int64_t)d * a.states + n] * kLog2e : 0.0f;
  float st = 0.0f;
  constexpr int R = 16;  // loads under way
  for (int64_t j0 = 0; j0 < segments; j0 += R) {
    float e[R], s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t j = min(j0 + r, segments - 1), k = BACK ? segments - 1 - j : j;
      e[r] = a.seg_state[k * n_all + i];
      s[r] = a.seg_reach[k * a.dim + d];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t j = j0 + r, k = BACK ? segments - 1 - j : j;
      if (j >= segments) continue;
      a.seg_start[k * n_all + i] = st;
      st = s[r] < 0.0f ? e[r] : carried(a2, s[r], st) + e[r];
    }
  }
}

template <int CTRL>
__device__ inline float moved(float v) {  // of the lane that CTRL says, in the same 16 lanes
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140, kTurn8 = 0x128, kAhead4 = 0x104;

// sum over the LPC lanes that share an element, the same in all of them
template <int LPC>
__device__ inline float lane_sum(float v) {
  v += moved<kSwap1>(v);
  v += moved<kSwap2>(v);
  if constexpr (LPC >= 8) v += moved<kMirror8>(v);
  if constexpr (LPC >= 16) v += moved<kMirror16>(v);
  return v;
}

// Sums over the elements of a wavefront of 8 numbers a lane (db and dc of four states), to LDS: with each step half of the numbers go to
// half of the lanes, by exchanges of halves and of 16 lanes between two registers.
template <int HALF>
__device__ inline void halve32(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < HALF; ++i) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v[i]), __builtin_bit_cast(unsigned, v[i + HALF]), false, false);
    const unsigned low = r[0], high = r[1];  // (a cast of the element itself is compiled to one of the first, ROCm 7.2)
    v[i] = __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
  }
}
template <int HALF>
__device__ inline void halve16(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < HALF; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v[i]), __builtin_bit_cast(unsigned, v[i + HALF]), false, false);
    const unsigned low = r[0], high = r[1];
    v[i] = __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
  }
}
// where lane `lane` has its numbers after that: place of the first one of a row's 2 NP, and whether they are another lane's too
template <int NP>
__device__ inline int place_of(int lane) {
  constexpr int LPC = NP / 4;
  int m = (lane & 32 ? 4 : 0) + (lane & 16 ? 2 : 0);
  if (LPC <= 8) m += lane & 8 ? 1 : 0;
  return (m >= 4 ? NP : 0) + 4 * (lane % LPC) + (m & 3);
}
template <int NP>
__device__ inline void sum_elements(float (&v)[8], float *to, bool up8) {
  constexpr int LPC = NP / 4;
  halve32<4>(v);
  halve16<2>(v);
  if constexpr (LPC <= 8) {
    const float keep = up8 ? v[1] : v[0], send = up8 ? v[0] : v[1];
    v[0] = keep + moved<kTurn8>(send);
    if constexpr (LPC == 4) v[0] += moved<kAhead4>(v[0]);  // in the lanes that give
    to[0] = v[0];
  } else {
    to[0] = v[0];
    to[1] = v[1];
  }
}

// The kernel's arguments, read again: kept in scalar registers through a loop there would be more of them than there are, and each use of one that has
// been moved to a vector register's lane is a vector instruction.
using ArgsInPlace = const __attribute__((address_space(4))) SsmArgs;
__device__ inline ArgsInPlace *args_again() {
  ArgsInPlace *p = (ArgsInPlace *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

// Backward of a unit's rows: a lane has states 4 q .. 4 q + 3 of an element; a workgroup's wavefronts have elements side by side.  Rows are gone
// through in blocks of kSaved, last block first, each bag's rows of a block at a time: forward from the state before them, w and
// the decays kept in registers, and back.
template <class E, int NP, int WAVES, bool GATED>
__global__ __launch_bounds__(64 * WAVES, 2) void ssm_grad_kernel(SsmArgs a) {
  constexpr int S = kSaved, LPC = NP / 4, CPW = 64 / LPC, OWN = (S + LPC - 1) / LPC;  // lanes of an element, elements of a wavefront, rows whose scalars a lane finds
  constexpr int V = 16 / sizeof(E), CH = CPW * WAVES, THREADS = 64 * WAVES;           // elements and lanes of a workgroup
  constexpr int PACKS = CH / V, BRINGS = (4 * S * PACKS + THREADS - 1) / THREADS;     // of a row; of x, delta, dy and z of a block that a lane brings
  constexpr int NUMBERS = (S * 2 * NP + THREADS - 1) / THREADS;                       // of b and c
  __shared__ Words<E, V> tile[2][4][S][PACKS];
  __shared__ float bc[2][S][2 * NP], part[2][WAVES][S][2 * NP];
  __shared__ float4 rows_of[WAVES][S][CPW];  // D, D x, dv, x
  __shared__ float spare[S][2 * NP];         // for the lanes whose sums are another lane's: a store that all lanes make needs no branch
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, q = lane % LPC, e = lane / LPC, N = a.states;
  float4(*row)[CPW] = rows_of[wave];
  const int place = place_of<NP>(lane);
  const bool up8 = lane & 8, give = LPC != 4 || !(lane & 4);
  const int64_t worker = blockIdx.x / a.blocks;
  const int block = (int)(blockIdx.x % a.blocks), d = block * CH + wave * CPW + e, dc = min(d, a.dim - 1);
  const bool in = d < a.dim, with_h0 = a.h0, with_dlast = a.dlast;
  const int group = a.groups > 1 ? block * CH / (a.dim / a.groups) : 0;
  float av[4], da[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dskip = 0.0f, dbias = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) av[j] = 4 * q + j < N ? a.a[(int64_t)dc * N + 4 * q + j] : 0.0f;
  const float bias = a.bias ? a.bias[dc] : 0.0f, skip = a.skip ? a.skip[dc] : 0.0f;
  const bool even = N % 4 == 0;  // the states of a lane are all there, or none
  // four states of [.., dim, states] numbers, to be waited for; nothing beyond the states
  auto four = [&](const float *p, float (&to)[4]) {
    if (even) {
      const int at = 4 * q < N ? 4 * q : 0;
      load_floats<float, 4>(p + (int64_t)dc * N + at, 4, to);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = p[(int64_t)dc * N + min(4 * q + j, N - 1)];
    }
  };
  auto known = [&](bool there, const float (&from)[4], float (&to)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = there && 4 * q + j < N ? from[j] : 0.0f;
  };

  // The blocks of this workgroup's units one after the other: units side by side, because what one of them has more its neighbour has less.
  const int64_t past = (worker + 1) * a.count / a.workers;
  struct Place {
    int64_t row0, begin, end, k;
    bool there;
  };
  auto enter = [&](int64_t k) {
    const auto &a = *args_again();
    for (; k < past; ++k) {
      const int64_t begin = a.units[k].begin, end = a.units[k + 1].begin;
      if (begin < end) return Place{(end - 1) & ~(int64_t)(S - 1), begin, end, k, true};
    }
    return Place{0, 0, 1, k, false};  // (what is read ahead of it is not used)
  };
  auto after = [&](Place p) {
    if (p.there && p.row0 <= p.begin) return enter(p.k + 1);
    p.row0 = max(p.row0 - S, (int64_t)0);
    return p;
  };
  // What a lane brings of a block, one block ahead: packs of the inputs (this lane's are all of one kind), numbers of b and c, the states before it; marks two
  // blocks ahead, so that the states at the end of its last bag are there too.
  Words<E, V> raw[BRINGS];
  E shared[NUMBERS];
  float4 before;
  auto fetch = [&](const Place &p) {
    const int me = lane_again();
    const auto &a = *args_again();
#pragma unroll
    for (int i = 0; i < BRINGS; ++i) {
      const int n = me + i * THREADS, kind = n / (S * PACKS) & 3, t = n / PACKS % S, at = block * CH + n % PACKS * V;
      const E *from = (const E *)(kind == 0 || (kind == 3 && !GATED) ? a.x : kind == 1 ? a.delta : kind == 2 ? a.dy : a.z);
      const int64_t stride = kind == 0 || (kind == 3 && !GATED) ? a.xs : kind == 1 ? a.ts : kind == 2 ? a.dys : a.zs;
      load_pack_of<E, V>(from + min(max(p.row0 + t, p.begin), p.end - 1) * stride, a.dim, at, raw[i]);
    }
#pragma unroll
    for (int i = 0; i < NUMBERS; ++i) {
      const int n = me + i * THREADS, t = n / (2 * NP) % S, m = n % (2 * NP);
      const int64_t r = min(max(p.row0 + t, p.begin), p.end - 1);
      const E *from = m < NP ? (const E *)a.b + r * a.bs : (const E *)a.c + r * a.cs;
      shared[i] = from[group * N + min(m % NP, N - 1)];
    }
    before = *(const float4 *)(a.saved + (p.row0 / S * a.dim + dc) * NP + 4 * q);
  };
  auto mark_at = [&](const Place &p) { return args_again()->marks[min(max(p.row0 + (lane & (S - 1)), p.begin), p.end - 1)]; };
  // a block's rows that are this unit's, and the bags that start and end in them
  struct Seen {
    int lo, hi;
    uint32_t starts, ends;
  };
  auto look = [&](const Place &p, int2 mark) {
    Seen s;
    s.lo = (int)max(p.begin - p.row0, (int64_t)0), s.hi = (int)min(p.end - p.row0, (int64_t)S);
    const bool mine = lane >= s.lo && lane < s.hi;
    s.starts = (uint32_t)__ballot(mine && mark.x >= 0), s.ends = (uint32_t)__ballot(mine && mark.y >= 0);
    return s;
  };
  // states that the last bag's rows [from, to) of [.., to) begin with, and gradients that they end with, if it starts and ends there
  struct Bag {
    int from;
    bool starts, ends;
  };
  auto last_bag = [&](const Seen &s, int to) {
    const uint32_t b = s.starts & ((1u << to) - 1);
    return Bag{b ? 31 - __builtin_clz(b) : s.lo, b != 0, (s.ends >> (to - 1) & 1) != 0};
  };
  auto ask = [&](const Bag &b, int to, int2 mark, float (&h)[4], float (&g)[4]) {
    const auto &a = *args_again();
    if (b.starts && a.h0) four(a.h0 + (int64_t)__builtin_amdgcn_readlane(mark.x, b.from) * a.h0s, h);
    if (b.ends && a.dlast) four(a.dlast + (int64_t)__builtin_amdgcn_readlane(mark.y, to - 1) * a.dim * N, g);
  };
  // db and dc of a block, from the wavefronts' sums
  auto give_shared = [&](const Place &p, int buffer) {
    const int me = lane_again();
    const auto &a = *args_again();
#pragma unroll
    for (int i = 0; i < NUMBERS; ++i) {
      const int n = me + i * THREADS, t = n / (2 * NP), m = n % (2 * NP), s = m % NP;
      const int64_t r = p.row0 + t;
      if (t >= S || r < p.begin || r >= p.end || s >= N) continue;
      float v = 0.0f;
#pragma unroll
      for (int j = 0; j < WAVES; ++j) v += part[buffer][j][t][m];
      if (a.shared) a.shared[((int64_t)block * a.rows + r) * 2 * N + (m < NP ? 0 : N) + s] = v;
      else ((E *)(m < NP ? a.db : a.dc))[r * a.groups * N + group * N + s] = (E)v;
    }
  };

  Place now = enter(worker * a.count / a.workers), done{0, 0, 0, 0, false};
  if (now.there) {
    Place next = after(now);
    int2 mark = mark_at(now), mark_next = mark_at(next);
    fetch(now);
    Seen seen = look(now, mark);
    Bag bag = last_bag(seen, seen.hi);
    float carry[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // exp(D a) g of the row behind
    float asked_h[4] = {0.0f, 0.0f, 0.0f, 0.0f}, asked_g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    ask(bag, seen.hi, mark, asked_h, asked_g);
    int64_t unit = -1;
    int buffer = 0;
    do {
      const Place then = after(next);
#pragma unroll
      for (int i = 0; i < BRINGS; ++i) {
        const int n = threadIdx.x + i * THREADS;
        if (4 * S * PACKS % THREADS == 0 || n < 4 * S * PACKS) (&tile[buffer][0][0][0])[n] = raw[i];
      }
#pragma unroll
      for (int i = 0; i < NUMBERS; ++i) {
        const int n = threadIdx.x + i * THREADS;
        if (S * 2 * NP % THREADS == 0 || n < S * 2 * NP) (&bc[buffer][0][0])[n] = n % NP < N ? (float)shared[i] : 0.0f;
      }
      const float saved[4] = {before.x, before.y, before.z, before.w};
      const Seen here = seen;
      const int2 bag_of = mark;
      const Bag first = bag;
      fetch(next);
      mark = mark_next;
      mark_next = mark_at(then);
      seen = look(next, mark);
      bag = last_bag(seen, seen.hi);
      __syncthreads();
      if (done.there) give_shared(done, buffer ^ 1);
      if (now.k != unit) {
        unit = now.k;
#pragma unroll
        for (int j = 0; j < 4; ++j) carry[j] = 0.0f;
        if (args_again()->units[unit + 1].cut) {
          const float a2[4] = {av[0] * kLog2e, av[1] * kLog2e, av[2] * kLog2e, av[3] * kLog2e};
          start_of<NP>(a, unit, dc, 4 * q, a2, carry);
          settle(carry);
        }
      }
      // scalars of the rows t with t % LPC = q
      float slope[OWN], gate[OWN], own_v[OWN], own_b[OWN], own_w[OWN];
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const int t = min(i * LPC + q, S - 1), at = t * CH + wave * CPW + e;
        const E *in_x = (const E *)tile[buffer] + at;
        constexpr int of = S * CH;
        // elements beyond the row (of which there is nothing in the tile) have no part of db and dc
        const float u = (in ? (float)in_x[of] : 0.0f) + bias, dy = in ? (float)in_x[2 * of] : 0.0f, step = soft(u), x = in ? (float)in_x[0] : 0.0f;
        float dv = dy;
        slope[i] = sigmoid(u);
        gate[i] = 0.0f;
        if (GATED) {
          const float z = in ? (float)in_x[3 * of] : 0.0f, f = sigmoid(z);
          dv = dy * z * f;
          gate[i] = dy * (f * (1.0f + z * (1.0f - f)));
        }
        own_v[i] = own_b[i] = own_w[i] = 0.0f;
        if (i * LPC + q < S) row[i * LPC + q][e] = make_float4(step, step * x, dv, x);
      }
      float *sums = (give ? &part[buffer][wave][0][0] : &spare[0][0]) + place;
      // the bags' rows [from, to) of the block, from the last
      Bag rows = first;
      for (int to = here.hi; to > here.lo;) {
        float h[4], w[S][4], decay[S][4];
        if (to != here.hi) {
          rows = last_bag(here, to);
          ask(rows, to, bag_of, asked_h, asked_g);
        }
        const int from = rows.from;
        float start[4], finish[4];
        known(with_h0, asked_h, start);
        known(with_dlast, asked_g, finish);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = rows.starts ? start[j] : saved[j];  // (a unit that begins within a block begins with a bag)
#pragma unroll
        for (int j = 0; j < 4; ++j) carry[j] = rows.ends ? finish[j] : carry[j];
        settle(h);
        settle(carry);
        if (from <= here.lo) ask(bag, seen.hi, mark, asked_h, asked_g);  // the next block's, while this one's last rows are gone through
        // Whole blocks apart: without branches between them, rows are interleaved, which hides the way through LDS and the chains of exchanges.
        auto walk = [&](auto whole) {
          constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
          for (int t = 0; t < S; ++t) {
            if (!WHOLE && (t < from || t >= to)) continue;
            if (WHOLE && t % 2 == 0) __builtin_amdgcn_sched_barrier(0);  // more rows at once do not fit the registers
            const float4 s = row[t][e], b = *(const float4 *)&bc[buffer][t][4 * q];
            const float bj[4] = {b.x, b.y, b.z, b.w};
            const float s2 = s.x * kLog2e;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              decay[t][j] = __builtin_amdgcn_exp2f(s2 * av[j]);
              w[t][j] = decay[t][j] * h[j];
              h[j] = w[t][j] + s.y * bj[j];
            }
            if (GATED) {
              const float4 c = *(const float4 *)&bc[buffer][t][NP + 4 * q];
              const float v = lane_sum<LPC>((c.x * h[0] + c.y * h[1]) + (c.z * h[2] + c.w * h[3]));
              own_v[t / LPC] = t % LPC == q ? v : own_v[t / LPC];
            }
          }
#pragma unroll
          for (int t = S - 1; t >= 0; --t) {
            if (!WHOLE && (t < from || t >= to)) continue;
            if (WHOLE && t % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            const float4 s = row[t][e], b = *(const float4 *)&bc[buffer][t][4 * q], c = *(const float4 *)&bc[buffer][t][NP + 4 * q];
            const float bj[4] = {b.x, b.y, b.z, b.w}, cj[4] = {c.x, c.y, c.z, c.w};
            float gb = 0.0f, gwa = 0.0f, both[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float g = cj[j] * s.z + carry[j], gw = g * w[t][j];
              gb += g * bj[j];
              gwa += gw * av[j];
              da[j] += gw * s.x;
              both[j] = g * s.y;
              both[4 + j] = s.z * (w[t][j] + s.y * bj[j]);
              carry[j] = decay[t][j] * g;
            }
            gb = lane_sum<LPC>(gb);
            gwa = lane_sum<LPC>(gwa);
            own_b[t / LPC] = t % LPC == q ? gb : own_b[t / LPC];
            own_w[t / LPC] = t % LPC == q ? gwa : own_w[t / LPC];
            sum_elements<NP>(both, sums + t * 2 * NP, up8);
          }
        };
        if (from == 0 && to == S) walk(std::true_type{});
        else walk(std::false_type{});
        if (rows.starts && args_again()->dh0) {
          const int64_t first_bag = __builtin_amdgcn_readlane(bag_of.x, from);  // by all lanes, as everywhere: the lane that knows may be beyond the row
          if (in) store_floats<float, 4>(args_again()->dh0 + (first_bag * args_again()->dim + d) * N + 4 * q, N - 4 * q, carry);
        }
        to = from;
      }
      const int me = lane_again() & 63;
      const auto &again = *args_again();
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const int t = i * LPC + me % LPC, of = block * CH + wave * CPW + me / LPC;
        if (t < here.lo || t >= here.hi || of >= again.dim) continue;
        const int64_t at = (now.row0 + t) * again.dim + of;
        const float4 s = row[t][me / LPC];
        const float du = (own_w[i] + s.w * own_b[i]) * slope[i];
        ((E *)again.dx)[at] = (E)(skip * s.z + s.x * own_b[i]);
        ((E *)again.ddelta)[at] = (E)du;
        if (GATED) ((E *)again.dz)[at] = (E)(gate[i] * (own_v[i] + skip * s.w));
        dskip += s.z * s.w;
        dbias += du;
      }
      done = now;
      now = next;
      next = then;
      buffer ^= 1;
    } while (now.there);
    __syncthreads();
    give_shared(done, buffer ^ 1);
  }
  dskip = lane_sum<LPC>(dskip);
  dbias = lane_sum<LPC>(dbias);
  if (!in) return;
  float *to = a.parts + (worker * a.dim + d) * (N + 2);
  store_floats<float, 4>(to + 4 * q, N - 4 * q, da);
  if (q == 0) to[N] = dskip, to[N + 1] = dbias;
}

// db and dc from the sums of the workgroups that a group's elements lie on
template <class E>
__global__ __launch_bounds__(kThreads) void ssm_shared_kernel(SsmArgs a, int64_t first) {
  const int64_t i = first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int N = a.states, width = 2 * N, of_group = a.blocks / a.groups;
  const int64_t r = i / (width * a.groups);
  if (r >= a.rows) return;
  const int k = (int)(i % (width * a.groups)), group = k / width, n = k % width;
  float v = 0.0f;
  for (int j = 0; j < of_group; ++j) v += a.shared[((int64_t)(group * of_group + j) * a.rows + r) * width + n];
  ((E *)(n < N ? a.db : a.dc))[(r * a.groups + group) * N + n % N] = (E)v;
}

// One more row: LPC lanes with four states each for an element
template <class E, int NP>
__global__ __launch_bounds__(kThreads) void ssm_step_kernel(SsmArgs a, float *state, int64_t stride, int64_t slots, const int64_t *slot_of, int64_t first) {
  constexpr int LPC = NP / 4;
  const int N = a.states;
  const int64_t i = first + ((int64_t)blockIdx.x * kThreads + threadIdx.x) / LPC, r = i / a.dim;
  if (r >= a.rows) return;  // all lanes of an element
  const int d = (int)(i - r * a.dim), q = threadIdx.x % LPC;
  const int64_t slot = slot_of ? slot_of[r] : r;
  float v = 0.0f;
  if (slot >= 0 && slot < slots) {
    float *s = state + slot * stride + (int64_t)d * N + 4 * q;
    const int have = N - 4 * q;
    float h[4], av[4], b[4], c[4];
    load_floats<float, 4>(s, have, h);
    load_floats<float, 4>(a.a + (int64_t)d * N + 4 * q, have, av);
    const int at = (a.groups > 1 ? d / (a.dim / a.groups) : 0) * N + 4 * q;
    load_floats<E, 4>((const E *)a.b + r * a.bs + at, have, b);
    load_floats<E, 4>((const E *)a.c + r * a.cs + at, have, c);
    const float x = (float)((const E *)a.x)[r * a.xs + d];
    const float step = soft((float)((const E *)a.delta)[r * a.ts + d] + (a.bias ? a.bias[d] : 0.0f));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      h[j] = __builtin_amdgcn_exp2f(step * (av[j] * kLog2e)) * h[j] + (step * x) * b[j];
      if (j < have) v += c[j] * h[j];
    }
    store_floats<float, 4>(s, have, h);
    v = lane_sum<LPC>(v);
    if (a.skip) v += a.skip[d] * x;
    if (a.z) {
      const float z = (float)((const E *)a.z)[r * a.zs + d];
      v *= z * sigmoid(z);
    }
  } else if (slot >= slots && q == 0) {
    *a.err = 2;
  }
  if (a.y && q == 0) ((E *)a.y)[r * a.ys + d] = (E)v;
}

// How the rows are cut: a function of their number and dim, so that forward and backward do the same.  As few cuts as leave 8192 wavefronts
// (eight a SIMD), down to 32 rows a unit.
int unit_of(int64_t rows, int dim) {
  int unit = 128;
  while (unit > 32 && divide_up(rows, unit) * divide_up(dim, 64) < 8192) unit /= 2;
  return unit;
}
int padded(int states) { return states <= 16 ? 16 : states <= 32 ? 32 : 64; }

// How the elements of a row lie on the backward's workgroups
struct GradLay {
  int waves, blocks;  // of a workgroup; workgroups of a row
};
GradLay grad_lay(int dim, int groups, int np) {
  const int each = 64 / (np / 4);  // elements of a wavefront
  const bool eight = groups > 1 ? dim / groups % (8 * each) == 0 : dim > 4 * each;  // a workgroup's elements are of one group
  const int waves = eight ? 8 : 4;
  return {waves, (int)divide_up(dim, waves * each)};
}
int64_t workers_of(int64_t units, GradLay l) { return std::max<int64_t>(1, std::min<int64_t>(units, kGradWaves / l.waves / l.blocks)); }

}  // namespace

struct tbe_ssm_t : DenseBase {
  int dim, states, groups, dtype, np;
  int64_t max_bags, max_rows;
  char *block = nullptr;
  int32_t *err;
  SsmArgs scratch{};
};

namespace {

int64_t most_units(int64_t rows, int dim) {  // of any number of rows up to this
  return std::max(divide_up(rows, unit_of(rows, dim)), std::min(divide_up(rows, 32), divide_up(8192, divide_up(dim, 64)) * 2 + 1));
}

template <int NP, bool BACK>
void join(const SsmArgs &a, hipStream_t st) {
  const int64_t segments = divide_up(a.count, kSegment), groups = divide_up((int64_t)a.dim * NP, kThreads);
  ssm_join_kernel<NP, BACK><<<dim3((unsigned)(segments * groups)), kThreads, 0, st>>>(a, segments, (int)groups);
  ssm_segments_kernel<NP, BACK><<<dim3((unsigned)divide_up((int64_t)a.dim * NP, 64)), 64, 0, st>>>(a, segments);
}

void prepare(const SsmArgs &a, float *empty_to, const float *empty_from, int64_t stride, hipStream_t st) {
  const int64_t bag_groups = divide_up(a.bags, kThreads), groups = bag_groups + divide_up(a.count + 1, kThreads / 64);  // (the unit behind the last: an end)
  ssm_prepare_kernel<<<dim3((unsigned)groups), kThreads, 0, st>>>(a, bag_groups, empty_to, empty_from, stride);
}

template <class E, int NP>
int forward(const SsmArgs &a, hipStream_t st) {
  prepare(a, a.last, a.h0, a.h0s, st);
  if (a.rows > 0) {
    const dim3 grid((unsigned)(a.count * a.waves));
    if (a.rows > 2 * a.unit) {  // else no bag is cut
      ssm_ends_kernel<E, NP, false><<<grid, 64, 0, st>>>(a);
      join<NP, false>(a, st);
    }
    if (a.states == NP) ssm_kernel<E, NP, true><<<grid, 64, 0, st>>>(a);
    else ssm_kernel<E, NP, false><<<grid, 64, 0, st>>>(a);
  }
  return check_launch();
}

template <class E, int NP>
int backward(SsmArgs a, const tbe_ssm_grads *g, hipStream_t st) {
  prepare(a, a.dh0, a.dlast, (int64_t)a.dim * a.states, st);
  const GradLay l = grad_lay(a.dim, a.groups, NP);
  a.blocks = l.blocks;
  a.workers = workers_of(a.count, l);
  if (l.blocks / a.groups <= 1) a.shared = nullptr;
  if (a.rows > 2 * a.unit) {
    ssm_ends_kernel<E, NP, true><<<dim3((unsigned)(a.count * a.waves)), 64, 0, st>>>(a);
    join<NP, true>(a, st);
  }
  const dim3 grid((unsigned)(a.workers * l.blocks));
  if (l.waves == 8) a.z ? ssm_grad_kernel<E, NP, 8, true><<<grid, 512, 0, st>>>(a) : ssm_grad_kernel<E, NP, 8, false><<<grid, 512, 0, st>>>(a);
  else a.z ? ssm_grad_kernel<E, NP, 4, true><<<grid, 256, 0, st>>>(a) : ssm_grad_kernel<E, NP, 4, false><<<grid, 256, 0, st>>>(a);
  if (a.shared) {
    const int64_t groups = divide_up(a.rows * a.groups * 2 * a.states, kThreads);
    for (int64_t done = 0; done < groups; done += most_groups(kThreads))
      ssm_shared_kernel<E><<<dim3((unsigned)std::min(groups - done, most_groups(kThreads))), kThreads, 0, st>>>(a, done * kThreads);
  }
  sum_parts(a.parts, a.workers, (int64_t)a.dim * (a.states + 2), a.states + 2, a.states, g->d_da, g->d_dskip, g->d_ddelta_bias, st);
  return check_launch();
}

template <class E, int NP>
int step(const SsmArgs &a, float *state, int64_t stride, int64_t slots, const int64_t *slot_of, hipStream_t st) {
  constexpr int each = kThreads / (NP / 4);  // elements of a workgroup
  const int64_t groups = divide_up(a.rows * a.dim, each);
  for (int64_t done = 0; done < groups; done += most_groups(kThreads))
    ssm_step_kernel<E, NP><<<dim3((unsigned)std::min(groups - done, most_groups(kThreads))), kThreads, 0, st>>>(a, state, stride, slots, slot_of, done * each);
  return check_launch();
}

// call<E, NP>() for the handle's type and number of states
template <class E, class F>
int of_states(int np, F call) {
  return np == 16 ? call.template operator()<E, 16>() : np == 32 ? call.template operator()<E, 32>() : call.template operator()<E, 64>();
}
template <class F>
int of_handle(tbe_ssm_handle s, F call) {
  if (s->dtype == TBE_FP32) return of_states<float>(s->np, call);
  if (s->dtype == TBE_FP16) return of_states<_Float16>(s->np, call);
  return of_states<__bf16>(s->np, call);
}
struct Forward {
  SsmArgs a;
  hipStream_t st;
  template <class E, int NP> int operator()() const { return forward<E, NP>(a, st); }
};
struct Backward {
  SsmArgs a;
  const tbe_ssm_grads *g;
  hipStream_t st;
  template <class E, int NP> int operator()() const { return backward<E, NP>(a, g, st); }
};
struct Step {
  SsmArgs a;
  float *state;
  int64_t stride, slots;
  const int64_t *slot_of;
  hipStream_t st;
  template <class E, int NP> int operator()() const { return step<E, NP>(a, state, stride, slots, slot_of, st); }
};

int check_batch(tbe_ssm_handle s, const tbe_ssm_batch *b, bool bags) {
  if (int rc = check_handle(s)) return rc;
  if (!b) return report(TBE_EINVAL, "null batch");
  if (b->rows < 0 || (bags && b->bags < 0)) return report(TBE_EINVAL, "negative number of bags or rows");
  if (bags && (b->bags > s->max_bags || b->rows > s->max_rows)) return report(TBE_ELIMIT, "more bags or rows than the handle was created for");
  if (bags && b->bags == 0 && b->rows > 0) return report(TBE_EINVAL, "rows without a bag");
  if (bags && b->bags > 0 && !b->d_offsets) return report(TBE_EINVAL, "null offsets");
  if (!b->d_a || (b->rows > 0 && (!b->d_x || !b->d_delta || !b->d_b || !b->d_c))) return report(TBE_EINVAL, "null rows or decays");
  const int64_t k = (int64_t)s->groups * s->states;
  if (b->rows > 0 && (b->x_stride < s->dim || b->delta_stride < s->dim || (b->d_z && b->z_stride < s->dim) || b->b_stride < k || b->c_stride < k))
    return report(TBE_EINVAL, "a stride below the length of a row");
  if (bags && b->d_h0 && b->h0_stride != 0 && b->h0_stride < (int64_t)s->dim * s->states) return report(TBE_EINVAL, "a stride below the states of a bag");
  return TBE_OK;
}
// where a batch's inputs lie
struct Inputs {
  int64_t dim, states, rows, bags;
  int bytes;
  Span x, delta, z, b, c, a, skip, bias, offsets, h0;
  Inputs(tbe_ssm_handle s, const tbe_ssm_batch *t, bool with_bags = true)
      : dim(s->dim), states(s->states), rows(t->rows), bags(with_bags ? t->bags : 0), bytes(elem_bytes(s->dtype)) {
    const int64_t k = states * s->groups;
    x = rows_of(t->d_x, t->x_stride), delta = rows_of(t->d_delta, t->delta_stride), z = rows_of(t->d_z, t->z_stride);
    b = span(t->d_b, k, t->b_stride, rows, bytes), c = span(t->d_c, k, t->c_stride, rows, bytes);
    a = span(t->d_a, dim * states * 4), skip = span(t->d_skip, dim * 4), bias = span(t->d_delta_bias, dim * 4);
    offsets = with_bags ? span(t->d_offsets, (bags + 1) * 8) : Span{}, h0 = span(t->d_h0, dim * states, t->h0_stride, bags, 4);
  }
  Span rows_of(const void *p, int64_t stride) const { return span(p, dim, stride, rows, bytes); }
  Span of_bags(const void *p) const { return span(p, bags * dim * states * 4); }
  int apart(std::initializer_list<Span> written) const { return check_apart(written, {x, delta, z, b, c, a, skip, bias, offsets, h0}); }
};
SsmArgs args_of(tbe_ssm_handle s, const tbe_ssm_batch *b) {
  SsmArgs a = s->scratch;
  a.x = b->d_x, a.delta = b->d_delta, a.z = b->d_z, a.b = b->d_b, a.c = b->d_c;
  a.xs = b->x_stride, a.ts = b->delta_stride, a.zs = b->z_stride, a.bs = b->b_stride, a.cs = b->c_stride;
  a.a = b->d_a, a.skip = b->d_skip, a.bias = b->d_delta_bias, a.off = b->d_offsets, a.bags = b->bags, a.rows = b->rows;
  a.h0 = b->d_h0, a.h0s = b->h0_stride;
  a.dim = s->dim, a.states = s->states, a.groups = s->groups, a.err = s->err;
  a.unit = unit_of(b->rows, s->dim);
  a.count = divide_up(b->rows, a.unit);
  a.waves = (int)divide_up(s->dim, 64);
  return a;
}

}  // namespace

extern "C" {

int tbe_ssm_create(tbe_ssm_handle *out, int32_t dim, int32_t states, int32_t groups, int32_t dtype, int64_t max_bags, int64_t max_rows) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (dim < 1 || dim > 65536) return report(TBE_EINVAL, "dim outside 1 .. 65536");
  if (states < 1 || states > kMostStates) return report(TBE_EINVAL, "states outside 1 .. 64");
  if (groups < 1 || (groups > 1 && (dim % groups || dim / groups % 64))) return report(TBE_EINVAL, "groups: 1, or such that each has a multiple of 64 elements");
  if (!known_dtype(dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (max_bags < 0 || max_rows < 0) return report(TBE_EINVAL, "negative number of bags or rows");
  if (max_bags > (1ll << 38) / dim / states || max_rows > (1ll << 38) / dim || max_bags >= INT32_MAX)
    return report(TBE_ELIMIT, "more than 2^38 elements or states of bags, or 2^31 bags");
  const int np = padded(states);
  const int64_t units = most_units(max_rows, dim), segments = divide_up(units, kSegment), waves = divide_up(dim, 64);
  if (units * waves > most_groups(64) || segments * divide_up((int64_t)dim * np, kThreads) > most_groups(kThreads) ||
      divide_up(max_bags, kThreads) + divide_up(units + 1, kThreads / 64) > most_groups(kThreads))
    return report(TBE_ELIMIT, "more rows or bags than one launch can take");
  tbe_ssm_t *s = new (std::nothrow) tbe_ssm_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->dim = dim, s->states = states, s->groups = groups, s->dtype = dtype, s->np = np, s->max_bags = max_bags, s->max_rows = max_rows;
  const GradLay l = grad_lay(dim, groups, np);
  int64_t at = 256;
  auto take = [&](int64_t bytes) {
    const int64_t from = at;
    at += (bytes + 255) / 256 * 256;
    return from;
  };
  const int64_t o_units = take((units + 1) * sizeof(Unit)), o_marks = take(max_rows * sizeof(int2)), o_ends = take(units * dim * np * 4),
                o_spans = take(units * dim * 4), o_reach = take(units * dim * 4), o_state = take(segments * dim * np * 4),
                o_sreach = take(segments * dim * 4), o_start = take(segments * dim * np * 4), o_says = take(segments * 4),
                o_parts = take(workers_of(units, l) * dim * (states + 2) * 4),
                o_shared = take(l.blocks / groups > 1 ? (int64_t)l.blocks * max_rows * 2 * states * 4 : 0);
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&s->block, (size_t)at);
  if (e == hipSuccess) e = hipMemset(s->block, 0, 256);
  if (e != hipSuccess) {
    (void)hipFree(s->block);
    delete s;
    return report_hip(e);
  }
  s->err = (int32_t *)s->block;
  SsmArgs &a = s->scratch;
  a.units = (Unit *)(s->block + o_units), a.marks = (int2 *)(s->block + o_marks), a.ends = (float *)(s->block + o_ends);
  a.spans = (float *)(s->block + o_spans), a.reach = (float *)(s->block + o_reach), a.seg_state = (float *)(s->block + o_state);
  a.seg_says = (int32_t *)(s->block + o_says);
  a.seg_reach = (float *)(s->block + o_sreach), a.seg_start = (float *)(s->block + o_start), a.parts = (float *)(s->block + o_parts);
  a.shared = (float *)(s->block + o_shared);
  *out = s;
  return TBE_OK;
}

int tbe_ssm_destroy(tbe_ssm_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->block);
  delete s;
  return TBE_OK;
}

int64_t tbe_ssm_saved_floats(tbe_ssm_handle s, int64_t rows) {
  if (!s || rows < 0) return report(TBE_EINVAL, "null handle or a negative number of rows");
  return divide_up(rows, kSaved) * s->dim * s->np;
}

int tbe_ssm_forward(tbe_ssm_handle s, const tbe_ssm_batch *b, void *d_y, int64_t y_stride, float *d_last, float *d_saved, void *stream) {
  if (int rc = check_batch(s, b, true)) return rc;
  if (b->rows > 0 && !d_y) return report(TBE_EINVAL, "null results");
  if (b->rows > 0 && y_stride < s->dim) return report(TBE_EINVAL, "a stride below the length of a row");
  if ((uintptr_t)d_saved & 15) return report(TBE_EINVAL, "what is saved begins at no multiple of 16 bytes");
  const Inputs in(s, b);
  if (int rc = in.apart({in.rows_of(d_y, y_stride), in.of_bags(d_last), span(d_saved, tbe_ssm_saved_floats(s, b->rows) * 4)})) return rc;
  if (b->bags == 0) return TBE_OK;
  SsmArgs a = args_of(s, b);
  a.y = d_y, a.ys = y_stride, a.last = d_last, a.saved = d_saved;
  return of_handle(s, Forward{a, (hipStream_t)stream});
}

int tbe_ssm_backward(tbe_ssm_handle s, const tbe_ssm_batch *b, const float *d_saved, const tbe_ssm_grads *g, void *stream) {
  if (int rc = check_batch(s, b, true)) return rc;
  if (!g || !g->d_da) return report(TBE_EINVAL, "null gradients");
  if (b->rows > 0 && (!d_saved || !g->d_dy || !g->d_dx || !g->d_ddelta || !g->d_db || !g->d_dc || (b->d_z && !g->d_dz)))
    return report(TBE_EINVAL, "null pointer for what the forward saved or for a gradient");
  if ((uintptr_t)d_saved & 15) return report(TBE_EINVAL, "what is saved begins at no multiple of 16 bytes");
  if (b->rows > 0 && g->dy_stride < s->dim) return report(TBE_EINVAL, "a stride below the length of a row");
  const Inputs in(s, b);
  const int64_t shared = b->rows * s->groups * s->states * elem_bytes(s->dtype), each = (int64_t)s->dim * 4;
  const std::initializer_list<Span> written = {in.rows_of(g->d_dx, s->dim), in.rows_of(g->d_ddelta, s->dim), in.rows_of(b->d_z ? g->d_dz : nullptr, s->dim), span(g->d_db, shared),
                                               span(g->d_dc, shared), span(g->d_da, each * s->states), span(g->d_dskip, each), span(g->d_ddelta_bias, each), in.of_bags(g->d_dh0)};
  if (int rc = in.apart(written)) return rc;
  if (int rc = check_apart(written, {in.rows_of(g->d_dy, g->dy_stride), in.of_bags(g->d_dlast), span(d_saved, tbe_ssm_saved_floats(s, b->rows) * 4)})) return rc;
  SsmArgs a = args_of(s, b);
  a.saved = const_cast<float *>(d_saved), a.dy = g->d_dy, a.dys = g->dy_stride, a.dlast = g->d_dlast;
  a.dx = g->d_dx, a.ddelta = g->d_ddelta, a.dz = g->d_dz, a.db = g->d_db, a.dc = g->d_dc, a.dh0 = g->d_dh0;
  return of_handle(s, Backward{a, g, (hipStream_t)stream});
}

int tbe_ssm_step(tbe_ssm_handle s, const tbe_ssm_batch *b, float *d_state, int64_t state_stride, int64_t slots, const int64_t *d_slots, void *d_y,
                 int64_t y_stride, void *stream) {
  if (int rc = check_batch(s, b, false)) return rc;
  if (slots < 0) return report(TBE_EINVAL, "negative number of slots");
  if (b->rows > (1ll << 38) / s->dim / s->np) return report(TBE_ELIMIT, "more than 2^38 states");
  if (b->rows == 0) return TBE_OK;
  if (!d_state) return report(TBE_EINVAL, "null states");
  if (!d_slots && b->rows > slots) return report(TBE_EINVAL, "more rows than states");
  if (state_stride < (int64_t)s->dim * s->states || (d_y && y_stride < s->dim)) return report(TBE_EINVAL, "a stride below the length of a row or of a state");
  Inputs in(s, b, false);
  const Span y = in.rows_of(d_y, y_stride), state = span(d_state, (int64_t)s->dim * s->states, state_stride, slots, 4), of_rows = span(d_slots, b->rows * 8);
  if (int rc = in.apart({state})) return rc;
  if (int rc = check_apart({state, y}, {of_rows})) return rc;
  if (int rc = check_apart({state}, {y})) return rc;
  for (Span *r : {&in.x, &in.delta, &in.z})  // (an element's lanes read it before one of them writes there)
    if (same_span(*r, y)) *r = Span{};
  if (int rc = in.apart({y})) return rc;
  SsmArgs a = args_of(s, b);
  a.y = d_y, a.ys = y_stride;
  return of_handle(s, Step{a, d_state, state_stride, slots, d_slots, (hipStream_t)stream});
}

int tbe_ssm_check(tbe_ssm_handle s, void *stream) {
  if (int rc = check_handle(s)) return rc;
  return check_errors(s->err, (hipStream_t)stream);
}

}  // extern "C"
