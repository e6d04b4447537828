// Gated linear recurrence over the rows of every bag: forward, backward, one row for each of many states.
// Contract: include/tbe.h.
//
// A row maps the state h to a h + b, element by element, with a = f and b = (1 - f) x (or x); where a bag starts the state
// before does not count: a = 0, b = f h0 + ....  Two such maps, one after the other, are one again, (a2 a1, a2 b1 + b2), so the
// rows of all bags are cut into chunks of equal length wherever the bags begin, and no bag's length matters:
//   prepare  marks at the rows where bags start and end; the offsets are looked over  (scan_prepare_kernel)
//   sum      every chunk's map                                                   (scan_sum_kernel)
//   join     the states before the chunks, by a scan over the chunks' maps       (scan_join_kernel)
//   apply    every chunk's rows from the state before it                         (scan_apply_kernel, scan_grad_kernel)
// One chunk needs the last one only.  Where bags are short, most chunks have a start and so a state behind them that nothing before
// them has a part in: then there are no `sum` and `join`, and `apply` hears from the chunks before (behind) it, see hear_from.
// The gradient runs the other way with c_t = f_t g_t = f_t (dy_t + c_{t+1}), reset where a bag ends, beside the forward's states again
// from those before the chunks, which the forward saved.
//
// A row lies on L lanes of V elements (16 bytes, or the largest half of that, quarter, ... that divides dim), a lane has R rows in a row in
// registers, 32 elements of each input or fewer (apply_threads, grad_threads).  The maps of a wavefront's 64 / L lane groups are
// joined by exchange between lanes, those of the workgroup's wavefronts through LDS.
#include <algorithm>
#include <cmath>
#include <new>

#include "tbe_dense.h"
#include "tbe_internal.h"

using namespace tbe;

namespace {

#ifndef TBE_FIRST_CALL  // tests begin near the ends of the numbers
#define TBE_FIRST_CALL 1
#endif

constexpr int kThreads = 256, kWaves = kThreads / 64;
// A chunk's rows lie on as many lanes as leave four wavefronts a SIMD room for their registers: single elements and the gradient on more.
// (200000 rows of 33 in fp32, bags of 30: 67 + 77 us; with half the lanes 102 + 95.)
constexpr int apply_threads(int V) { return V <= 2 ? 2 * kThreads : kThreads; }
constexpr int grad_threads(int V) { return V <= 2 ? 4 * kThreads : 2 * kThreads; }
constexpr int64_t kChainedBags = 16;  // chunks that a bag may have on average for them to hear from each other
constexpr int kJoinChannels = 4, kJoinSegments = 256;

// How the rows of a handle are cut: a function of dim and the type alone, because the backward uses what the forward saved.
struct Cut {
  int V, R, L;  // elements and rows of a lane, lanes of a row (a power of two)
  int tiles;    // parts of L * V elements that a row has
  int rows;     // rows of a chunk
};

Cut cut_of(int dim, int dtype) {
  Cut c;
  c.V = 16 / elem_bytes(dtype);
  while (dim % c.V) c.V /= 2;
  c.R = 32 / c.V;
  const int lanes = dim / c.V;
  c.L = c.V == 1 ? 2 : 1;  // at least 2 for single elements: a chunk has 4096 rows at most
  while (c.L < lanes && c.L < 64) c.L *= 2;
  c.tiles = (lanes + c.L - 1) / c.L;
  c.rows = kThreads / c.L * c.R;
  return c;
}

// A map that does not depend on the state before it has a = -0: products with gates keep the sign, and joining maps leaves out what is
// before (0 times an infinity or a NaN of another bag would be a NaN).
constexpr float kReset = -0.0f;
__device__ inline void join(float pa, float ph, float &a, float &h) {  // (pa, ph) first, then (a, h)
  const bool reset = signbit(a);
  h = reset ? h : a * ph + h;
  a = reset ? a : a * pa;
}
__device__ inline float go(float a, float h, float s) { return signbit(a) ? h : a * s + h; }

// The two gates f = 1 / (1 + exp(-u)) and 1 - f in one number: the smaller one, negative where that is 1 - f.  Each then keeps
// its own bits (1 - f from a rounded f near one would not).  The exponential is the hardware's power of two of the rounded u log2(e), the constant
// itself in 32 bits, so a gate is off by up to (1.25 |u| + 8) 2^-24 of itself: 1.1e-6 at |u| = 8, 2.7e-6 at 30, where the gate is below 1e-13.  Carrying the product's rounding on
// would take 4 of some 32 (forward) and 83 (gradient) instructions an element more.
__device__ inline float gate(float u) {
  const float e = __builtin_amdgcn_exp2f(fabsf(u) * -1.44269504f), s = e * __builtin_amdgcn_rcpf(1.0f + e);
  return u >= 0.0f ? -s : s;
}
// f and (1 - f) x, or x
__device__ inline void gated(float u, float x, bool coupled, float &f, float &b) {
  const float e = __builtin_amdgcn_exp2f(u * -1.44269504f);  // infinite below u = -88
  f = __builtin_amdgcn_rcpf(1.0f + e);
  const float i = u < -80.0f ? 1.0f : e * f;
  b = coupled ? i * x : x;
}
__device__ inline float keep_of(float q) { return signbit(q) ? 1.0f - fabsf(q) : q; }
__device__ inline float take_of(float q) { return signbit(q) ? -q : 1.0f - fabsf(q); }

template <int DT>
struct Rows {
  using E = typename Elem<DT>::type;
  const E *x, *u, *dy;
  E *y, *dx, *du;
  int64_t xs, us, dys, ys, dxs, dus;
  const int64_t *off;
  const float *h0, *dlast;
  float *last, *dh0;
  float *maps;          // [chunks][2][dim]: a and b of the chunks
  float *before;        // [chunks][dim]: states before the chunks
  float *behind;        // [chunks][dim]: c behind the chunks
  uint64_t *words;      // [chunks][2][dim]: what chunks say to each other
  const ulonglong2 *marks;  // [rows]: call << 32 | the bag that starts at a row, and the same of the bag whose last row it is
  uint32_t *call;       // [0] number of this call, [1] of the next
  int64_t h0s, bags, rows;
  int dim, L, tiles, chunk_rows, chunks;
  bool coupled, chained;  // chained: chunks hear from each other instead of sum and join
};

// Numbers of calls: none whose 30 bits in a word are zero, as memory is that no call has written.  (What a chunk said 2^30 - 1 calls ago would
// pass for new, if no call since then had as many chunks and another one looks before it speaks.)
constexpr uint32_t kWordCall = 0x3FFFFFFFu;
__device__ inline uint32_t call_after(uint32_t call) { return (call + 1) & kWordCall ? call + 1 : call + 2; }

// V elements at any address that an element may have
template <class E, int V>
__device__ inline Pack<E, V> load_pack(const E *p) {
  Pack<E, V> r;
  __builtin_memcpy(&r, p, sizeof r);
  return r;
}
template <class E, int V>
__device__ inline void store_pack(E *p, const Pack<E, V> &r) {
  __builtin_memcpy(p, &r, sizeof r);
}

// Marks at the rows where bags start and end, with the number of the call (those of earlier calls are not cleared); empty bags get
// their last state (BACK: gradient of the first) here; offsets that do not ascend from 0 to rows are reported.
__global__ __launch_bounds__(kThreads) void scan_prepare_kernel(const int64_t *off, int64_t bags, int64_t rows, ulonglong2 *marks, uint32_t *call, int dim,
                                                                const float *from, int64_t stride, float *to, int32_t *err) {
  const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const uint32_t now = call[1];
  if (b == 0) call[0] = now;
  bool empty = false;
  if (b < bags) {
    const int64_t s = off[b], e = off[b + 1];
    if (s > e || s < 0 || e > rows || (b == 0 && s != 0) || (b == bags - 1 && e != rows)) {
      *err = 1;
    } else if (s == e) {
      empty = true;
    } else {
      const unsigned long long mark = (unsigned long long)now << 32 | (uint32_t)b;
      marks[s].x = mark;
      marks[e - 1].y = mark;
    }
  }
  if (!to) return;
  uint64_t todo = __ballot(empty);  // an empty bag at a time, by the whole wavefront
  while (todo) {
    const int64_t one = __shfl((int)b, __ffsll((unsigned long long)todo) - 1);
    for (int d = threadIdx.x & 63; d < dim; d += 64) to[one * dim + d] = from ? from[one * stride + d] : 0.0f;
    todo &= todo - 1;
  }
}

// The chunk's marks in LDS: [2 r] is 1 + the bag that starts at row r of the chunk, [2 r + 1] 1 + the bag whose last row that is, or 0.
template <int THREADS, class A>
__device__ inline void fetch_marks(const A &a, int64_t row0, uint32_t call, int32_t *marks) {
  for (int k = threadIdx.x; k < a.chunk_rows; k += THREADS) {
    const ulonglong2 m = row0 + k < a.rows ? a.marks[row0 + k] : ulonglong2{0, 0};
    marks[2 * k] = (uint32_t)(m.x >> 32) == call ? (int32_t)(uint32_t)m.x + 1 : 0;
    marks[2 * k + 1] = (uint32_t)(m.y >> 32) == call ? (int32_t)(uint32_t)m.y + 1 : 0;
  }
  __syncthreads();
}

// A word is a number with the call and what it is: the state behind (BACK: before) a chunk, or the b of its map, whose a is in the second
// word.  Each word says by itself whether it is there.
constexpr uint32_t kSaysMap = 1, kSaysState = 2;
__device__ inline uint64_t word_of(float v, uint32_t call, uint32_t kind) { return (uint64_t)(call << 2 | kind) << 32 | __float_as_uint(v); }
__device__ inline void put_word(uint64_t *p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Workgroups begin in the order of their numbers as a rule, but nothing waits for that: where a chunk has said nothing for as many looks as
// this, the rows of the bag are gone through from its start.
constexpr int kLooks = 16 * kPolls;  // a millisecond or so
__device__ inline bool get_word(const uint64_t *p, uint64_t &w, uint32_t call) {  // w: what a first look found
  for (int k = 0; (uint32_t)(w >> 34) != (call & kWordCall); k++) {
    if (k >= kLooks) return false;
    __builtin_amdgcn_s_sleep(1);
    w = look(p);
  }
  return true;
}

// The state before the chunk (BACK: behind it), for element d: from the nearest chunk that has said its state, through the maps of those in
// between, one after the other.  Every state that is said was found in this order too, so it has the same bits wherever it is found, but where a
// chunk has gone through the rows itself (walk_to): that one's order is another, and the last bits behind it may be.
template <bool BACK, class A>
__device__ inline bool hear_from(const A &a, int chunk, int d, uint32_t call, float &s) {
  constexpr int kAtOnce = 2;
  const int n = BACK ? a.chunks - 1 - chunk : chunk;  // chunks before this one; the first of them says its state and never a map
  s = 0.0f;
  if (n == 0) return true;
  const uint64_t *first = a.words + (int64_t)(BACK ? chunk + 1 : chunk - 1) * 2 * a.dim + d;
  const int64_t step = (BACK ? 2 : -2) * (int64_t)a.dim;
  int k = 0;  // chunks to go through
  for (bool found = false; !found;) {
    uint64_t w[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; q++) w[q] = look(first + min(k + q, n - 1) * step);
#pragma unroll
    for (int q = 0; q < kAtOnce; q++) {
      if (found) continue;
      if (!get_word(first + min(k, n - 1) * step, w[q], call)) return false;
      found = (w[q] >> 32 & 3) == kSaysState;
      s = __uint_as_float((uint32_t)w[q]);
      if (!found && ++k == n) return false;  // behind the first of them there are no words
    }
  }
  while (k > 0) {
    uint64_t h[kAtOnce], m[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; q++) {
      const uint64_t *p = first + max(k - 1 - q, 0) * step;
      h[q] = look(p);
      m[q] = look(p + a.dim);
    }
#pragma unroll
    for (int q = 0; q < kAtOnce; q++) {
      if (k == 0) continue;
      k--;
      if ((h[q] >> 32 & 3) == kSaysState) s = __uint_as_float((uint32_t)h[q]);
      else if (!get_word(first + k * step + a.dim, m[q], call)) return false;
      else s = go(__uint_as_float((uint32_t)m[q]), __uint_as_float((uint32_t)h[q]), s);
    }
  }
  return true;
}

// The same from the rows themselves, from the start (end) of the bag on.  Where a bag starts (ends) with the chunk, nothing asks for it.
template <bool BACK, class A>
__device__ float walk_to(const A &a, int chunk, int d, uint32_t call) {
  const int64_t row = (int64_t)(BACK ? chunk + 1 : chunk) * a.chunk_rows;  // the state before this row
  int64_t t = BACK ? row : row - 1;
  unsigned long long m;
  for (;; t += BACK ? 1 : -1) {
    m = BACK ? a.marks[t].y : a.marks[t].x;
    if ((uint32_t)(m >> 32) == call) break;
    if (BACK ? t + 1 >= a.rows : t <= 0) return 0.0f;
  }
  const int64_t b = (uint32_t)m;
  float s = BACK ? (a.dlast ? a.dlast[b * a.dim + d] : 0.0f) : (a.h0 ? a.h0[b * a.h0s + d] : 0.0f);
  for (; BACK ? t >= row : t < row; t += BACK ? -1 : 1) {
    const float q = gate((float)a.u[t * a.us + d]);
    if (BACK) s = keep_of(q) * ((a.dy ? (float)a.dy[t * a.dys + d] : 0.0f) + s);
    else s = keep_of(q) * s + (a.coupled ? take_of(q) : 1.0f) * (float)a.x[t * a.xs + d];
  }
  return s;
}

// What the chunk says of element d: its state where nothing before it has a part in that, else its map; then, told the state before it, the
// one behind it.  The first chunk has nothing before it, also where no bag starts in it (offsets that begin later) and where a NaN gate has
// taken the sign from its -0.  Returns the state before it.
template <bool BACK, class A>
__device__ inline float hear_and_say(const A &a, int chunk, int d, uint32_t call, float A1, float H1) {
  uint64_t *w = a.words + (int64_t)chunk * 2 * a.dim + d;
  const bool known = signbit(A1) || (BACK ? chunk == a.chunks - 1 : chunk == 0);
  if (known) {
    put_word(w, word_of(go(A1, H1, 0.0f), call, kSaysState));
  } else {
    put_word(w + a.dim, word_of(A1, call, kSaysMap));
    put_word(w, word_of(H1, call, kSaysMap));
  }
  float s;
  if (!hear_from<BACK>(a, chunk, d, call, s)) s = walk_to<BACK>(a, chunk, d, call);
  if (!known) put_word(w, word_of(go(A1, H1, s), call, kSaysState));
  return s;
}

// (A, H) becomes the map of all lane groups of the wavefront up to this one (BACK: from the last one down to it); reset: whether a bag starts
// (ends) among their rows, the same for all elements, so that what joins is a matter of lanes and not of each element.
template <int V, bool BACK>
__device__ inline void scan_wave(float (&A)[V], float (&H)[V], bool &reset, int L) {
  const int lane = threadIdx.x & 63;
  for (int k = L; k < 64; k *= 2) {
    float pa[V], ph[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      pa[v] = BACK ? __shfl_down(A[v], k) : __shfl_up(A[v], k);
      ph[v] = BACK ? __shfl_down(H[v], k) : __shfl_up(H[v], k);
    }
    const bool pr = BACK ? __shfl_down((int)reset, k) : __shfl_up((int)reset, k), has = BACK ? lane + k < 64 : lane >= k;
    if (has && !reset) {
#pragma unroll
      for (int v = 0; v < V; v++) {
        H[v] = A[v] * ph[v] + H[v];
        A[v] *= pa[v];
      }
      reset = pr;
    }
  }
}

// The wavefronts' maps go to LDS (tot: [kWaves][2][C]); map_of_waves, a lane for an element, has the map of all of them, join_waves leaves
// there the states before (behind) the wavefronts; start_of_lane goes on from there to that before (behind) the lane's rows.
template <int V, bool BACK>
__device__ inline void tell_wave(const float (&A)[V], const float (&H)[V], int L, float *tot) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, C = L * V, c = (lane & (L - 1)) * V;
  if (BACK ? lane < L : lane >= 64 - L)
#pragma unroll
    for (int v = 0; v < V; v++) {
      tot[(wave * 2) * C + c + v] = A[v];
      tot[(wave * 2 + 1) * C + c + v] = H[v];
    }
}
template <bool BACK, int W>
__device__ inline void map_of_waves(const float *tot, int C, int c, float &A, float &H) {
  A = 1.0f;
  H = 0.0f;
#pragma unroll
  for (int k = 0; k < W; k++) {
    const int w = BACK ? W - 1 - k : k;
    const float wa = tot[(w * 2) * C + c], wh = tot[(w * 2 + 1) * C + c];
    H = go(wa, wh, H);
    A = signbit(wa) ? wa : wa * A;
  }
}
template <bool BACK, int W>
__device__ inline void join_waves(float *tot, int C, int c, float s) {
#pragma unroll
  for (int k = 0; k < W; k++) {
    const int w = BACK ? W - 1 - k : k;
    const float wa = tot[(w * 2) * C + c], wh = tot[(w * 2 + 1) * C + c];
    tot[(w * 2) * C + c] = s;
    s = go(wa, wh, s);
  }
}
template <int V, bool BACK>
__device__ inline void start_of_lane(const float (&A)[V], const float (&H)[V], bool reset, int L, const float *tot, float (&s)[V]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, C = L * V, c = (lane & (L - 1)) * V;
  const bool first = BACK ? lane >= 64 - L : lane < L, pr = BACK ? __shfl_down((int)reset, L) : __shfl_up((int)reset, L);
#pragma unroll
  for (int v = 0; v < V; v++) {
    const float w = tot[(wave * 2) * C + c + v];
    const float pa = BACK ? __shfl_down(A[v], L) : __shfl_up(A[v], L), ph = BACK ? __shfl_down(H[v], L) : __shfl_up(H[v], L);
    s[v] = first ? w : pr ? ph : pa * w + ph;
  }
}

// V fp32 numbers of a row, or zeros without one
template <int V>
__device__ inline void load_row(const float *p, int64_t at, bool there, float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; k++) v[k] = p && there ? p[at + k] : 0.0f;
}

__device__ inline void opaque(float &x) { asm volatile("" : "+v"(x)); }

// Maps of the chunks: of h from x and u, BACK: of c from dy and u.  Bound by memory (3 bags of 100 k rows of 64 in fp32: 26 us, 6 TB/s).
template <int DT, int V, bool BACK>
__global__ __launch_bounds__(kThreads) void scan_sum_kernel(Rows<DT> a) {
  using E = typename Elem<DT>::type;
  constexpr int R = 32 / V;
  extern __shared__ float lds[];
  const int chunk = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, C = a.L * V;
  int32_t *marks = (int32_t *)(lds + kWaves * 2 * C);
  const int64_t row0 = (int64_t)chunk * a.chunk_rows;
  const int group = threadIdx.x / a.L, l = threadIdx.x & (a.L - 1), c0 = (tile * a.L + l) * V, r0 = group * R;
  const int rows = (int)min((int64_t)a.chunk_rows, a.rows - row0);
  const E *in = BACK ? a.dy : a.x;
  const int64_t stride = BACK ? a.dys : a.xs;
  Pack<E, V> xv[R], uv[R];
#pragma unroll
  for (int j = 0; j < R; j++) {
    const bool on = r0 + j < rows && c0 < a.dim;
    xv[j] = {};
    uv[j] = {};
    if (on) {
      uv[j] = load_pack<E, V>(a.u + (row0 + r0 + j) * a.us + c0);
      if (in) xv[j] = load_pack<E, V>(in + (row0 + r0 + j) * stride + c0);
    }
  }
  fetch_marks<kThreads>(a, row0, a.call[0], marks);
  float A[V], H[V];
  bool reset = false;
#pragma unroll
  for (int v = 0; v < V; v++) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int j = BACK ? R - 1 - k : k;
    const int32_t bag = marks[2 * (r0 + j) + (BACK ? 1 : 0)];
    if (bag) {
      reset = true;
      const float *s = BACK ? a.dlast : a.h0;
      const int64_t at = (int64_t)(bag - 1) * (BACK ? a.dim : a.h0s) + c0;
#pragma unroll
      for (int v = 0; v < V; v++) {
        A[v] = kReset;
        H[v] = s && c0 < a.dim ? s[at + v] : 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
      float f, b;
      gated((float)uv[j].e[v], (float)xv[j].e[v], !BACK && a.coupled, f, b);
      H[v] = BACK ? f * (H[v] + b) : f * H[v] + b;
      A[v] *= f;
    }
  }
  scan_wave<V, BACK>(A, H, reset, a.L);
  tell_wave<V, BACK>(A, H, a.L, lds);
  __syncthreads();
  for (int c = threadIdx.x; c < C && tile * C + c < a.dim; c += kThreads) {
    float A1, H1;
    map_of_waves<BACK, kWaves>(lds, C, c, A1, H1);
    a.maps[(int64_t)chunk * 2 * a.dim + tile * C + c] = A1;
    a.maps[((int64_t)chunk * 2 + 1) * a.dim + tile * C + c] = H1;
  }
}

// States before the chunks (BACK: behind them) from their maps.  A workgroup has 4 elements; its lanes take 256 segments of the chunks, up
// to kKept of each in registers, and a wavefront for each element joins the segments, 4 a lane, by exchange between lanes.  (With 16
// elements and 64 segments a workgroup there were too few lanes for the way to memory: 15.5 us instead of 11.9 for 2347 chunks of 64.)
template <bool BACK>
__global__ __launch_bounds__(kJoinChannels *kJoinSegments) void scan_join_kernel(const float *maps, float *state, int chunks, int dim) {
  constexpr int kKept = 8;
  __shared__ float tot[2][kJoinChannels][kJoinSegments];
  const int c = threadIdx.x % kJoinChannels, seg = threadIdx.x / kJoinChannels, d = blockIdx.x * kJoinChannels + c;
  const int per = (chunks + kJoinSegments - 1) / kJoinSegments, k0 = min(seg * per, chunks), k1 = min(k0 + per, chunks);
  const bool on = d < dim;
  auto at = [&](int k) { return (int64_t)(BACK ? chunks - 1 - k : k) * 2 * dim + d; };
  float A = 1.0f, H = 0.0f, ka[kKept], kh[kKept];
#pragma unroll
  for (int q = 0; q < kKept; q++) {
    ka[q] = on && k0 + q < k1 ? maps[at(k0 + q)] : 1.0f;
    kh[q] = on && k0 + q < k1 ? maps[at(k0 + q) + dim] : 0.0f;
  }
#pragma unroll
  for (int q = 0; q < kKept; q++) {
    H = go(ka[q], kh[q], H);
    A = signbit(ka[q]) ? ka[q] : ka[q] * A;
  }
  if (on)
#pragma unroll 8
    for (int k = k0 + kKept; k < k1; k++) {
      const float a = maps[at(k)], h = maps[at(k) + dim];
      H = go(a, h, H);
      A = signbit(a) ? a : a * A;
    }
  tot[0][c][seg] = A;
  tot[1][c][seg] = H;
  __syncthreads();
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (w < kJoinChannels) {
    constexpr int kEach = kJoinSegments / 64;
    float a[kEach], h[kEach], la = 1.0f, lh = 0.0f;
#pragma unroll
    for (int q = 0; q < kEach; q++) {
      a[q] = tot[0][w][lane * kEach + q];
      h[q] = tot[1][w][lane * kEach + q];
      lh = go(a[q], h[q], lh);
      la = signbit(a[q]) ? a[q] : a[q] * la;
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
      const float pa = __shfl_up(la, k), ph = __shfl_up(lh, k);
      if (lane >= k) join(pa, ph, la, lh);
    }
    float s = __shfl_up(lh, 1);
    s = lane ? s : 0.0f;
#pragma unroll
    for (int q = 0; q < kEach; q++) {
      tot[1][w][lane * kEach + q] = s;
      s = go(a[q], h[q], s);
    }
  }
  __syncthreads();
  if (!on) return;
  float s = tot[1][c][seg];
#pragma unroll
  for (int q = 0; q < kKept; q++) {
    if (k0 + q < k1) state[(int64_t)(BACK ? chunks - 1 - k0 - q : k0 + q) * dim + d] = s;
    s = go(ka[q], kh[q], s);
  }
#pragma unroll 8
  for (int k = k0 + kKept; k < k1; k++) {
    state[(int64_t)(BACK ? chunks - 1 - k : k) * dim + d] = s;
    s = go(maps[at(k)], maps[at(k) + dim], s);
  }
}

// The rows of a chunk, from the state before it.  x and u are read and y is written once; what starts a bag is taken into its first row's b, so
// the second way through the rows is one multiplication and addition an element.  Bound by memory where chunks need not hear from
// each other (3 bags of 100 k rows of 64 in fp32: 38 us, 6 TB/s), else half by vector instructions (32 an element), half by the way over two
// hand-overs in LDS and a word of another chunk (8192 bags of 30 rows of 128 in binary16: 46 us, 4.2 TB/s).
template <int DT, int V>
__global__ __launch_bounds__(apply_threads(V)) void scan_apply_kernel(Rows<DT> a) {
  using E = typename Elem<DT>::type;
  constexpr int T = apply_threads(V), W = T / 64, R = 32 * kThreads / T / V;
  extern __shared__ float lds[];
  const int chunk = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, C = a.L * V;
  int32_t *marks = (int32_t *)(lds + W * 2 * C);
  const int64_t row0 = (int64_t)chunk * a.chunk_rows;
  const int group = threadIdx.x / a.L, l = threadIdx.x & (a.L - 1), c0 = (tile * a.L + l) * V, r0 = group * R;
  const int rows = (int)min((int64_t)a.chunk_rows, a.rows - row0);
  const bool on = c0 < a.dim;
  Pack<E, V> xv[R], uv[R];
#pragma unroll
  for (int j = 0; j < R; j++) {
    xv[j] = {};
    uv[j] = {};
    if (on && r0 + j < rows) {
      uv[j] = load_pack<E, V>(a.u + (row0 + r0 + j) * a.us + c0);
      xv[j] = load_pack<E, V>(a.x + (row0 + r0 + j) * a.xs + c0);
    }
  }
  const uint32_t call = a.call[0];
  if (blockIdx.x == 0 && threadIdx.x == 0) a.call[1] = call_after(call);  // nothing looks at that one in this kernel
  fetch_marks<T>(a, row0, call, marks);
  // The first start among the lane's rows: its state is asked for before the gates are computed.
  int first = R;
#pragma unroll
  for (int j = R - 1; j >= 0; j--) first = marks[2 * (r0 + j)] ? j : first;
  float early[V];
  load_row(a.h0, first < R ? (int64_t)(marks[2 * (r0 + first)] - 1) * a.h0s + c0 : 0, first < R && on, early);
  float f[R][V], b[R][V], A[V], H[V];
#pragma unroll
  for (int j = 0; j < R; j++)
#pragma unroll
    for (int v = 0; v < V; v++) gated((float)uv[j].e[v], (float)xv[j].e[v], a.coupled, f[j][v], b[j][v]);
#pragma unroll
  for (int v = 0; v < V; v++) { A[v] = 1.0f; H[v] = 0.0f; }
  uint32_t starts = 0;
#pragma unroll
  for (int j = 0; j < R; j++) {
    const int32_t bag = marks[2 * (r0 + j)];
    if (bag) {  // what the bag starts from goes into b
      if (j != first) load_row(a.h0, (int64_t)(bag - 1) * a.h0s + c0, on, early);
      starts |= 1u << j;
#pragma unroll
      for (int v = 0; v < V; v++) {
        b[j][v] += f[j][v] * early[v];
        A[v] = kReset;
        H[v] = b[j][v];
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; v++) {
        H[v] = f[j][v] * H[v] + b[j][v];
        A[v] *= f[j][v];
      }
    }
  }
  bool reset = starts != 0;
  scan_wave<V, false>(A, H, reset, a.L);
  tell_wave<V, false>(A, H, a.L, lds);
  __syncthreads();
  for (int c = threadIdx.x; c < C; c += T) {
    const int d = tile * C + c;
    float s = 0.0f;
    if (a.chunks > 1 && d < a.dim) {
      float *before = a.before ? a.before + (int64_t)chunk * a.dim + d : nullptr;
      if (a.chained) {
        float A1, H1;
        map_of_waves<false, W>(lds, C, c, A1, H1);
        s = hear_and_say<false>(a, chunk, d, call, A1, H1);
        if (before) *before = s;
      } else {
        s = *before;
      }
    }
    join_waves<false, W>(lds, C, c, s);
  }
  __syncthreads();
  float h[V];
  start_of_lane<V, false>(A, H, reset, a.L, lds, h);
  if (!on) return;
#pragma unroll
  for (int j = 0; j < R; j++) {
    const int32_t ended = marks[2 * (r0 + j) + 1];
    Pack<E, V> out;
#pragma unroll
    for (int v = 0; v < V; v++) {
      h[v] = starts >> j & 1 ? b[j][v] : f[j][v] * h[v] + b[j][v];
      out.e[v] = (E)h[v];
    }
    if (a.y && r0 + j < rows) store_pack<E, V>(a.y + (row0 + r0 + j) * a.ys + c0, out);
    if (ended && a.last)
#pragma unroll
      for (int v = 0; v < V; v++) a.last[(int64_t)(ended - 1) * a.dim + c0 + v] = h[v];
  }
}

// The gradient of a chunk's rows: the states from that before it, c from that behind it, each joined like the forward's, then dx and du.  16
// elements a lane (8 where V is 1 or 2): with 32, as in the forward, two wavefronts a SIMD have room instead of four (120 us instead of 114 for 8192 bags of 30 rows of
// 128 in bfloat16, 80 instead of 75 for 3 bags of 100 k rows of 64 in fp32).  Bound by vector instructions, 83 an element, 0.6 of the time.
template <int DT, int V>
__global__ __launch_bounds__(grad_threads(V), 4) void scan_grad_kernel(Rows<DT> a) {
  using E = typename Elem<DT>::type;
  constexpr int T = grad_threads(V), W = T / 64, R = 32 * kThreads / T / V;
  extern __shared__ float lds[];
  // from the last chunk on: what a chunk hears of is behind it
  const int chunk = a.chunks - 1 - blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, C = a.L * V;
  float *back = lds + W * 2 * C;
  int32_t *marks = (int32_t *)(back + W * 2 * C);
  const int64_t row0 = (int64_t)chunk * a.chunk_rows;
  const int group = threadIdx.x / a.L, l = threadIdx.x & (a.L - 1), c0 = (tile * a.L + l) * V, r0 = group * R;
  const int rows = (int)min((int64_t)a.chunk_rows, a.rows - row0);
  const bool on = c0 < a.dim;
  Pack<E, V> xv[R], uv[R], gv[R];
#pragma unroll
  for (int j = 0; j < R; j++) {
    xv[j] = {};
    uv[j] = {};
    gv[j] = {};
    if (on && r0 + j < rows) {
      uv[j] = load_pack<E, V>(a.u + (row0 + r0 + j) * a.us + c0);
      xv[j] = load_pack<E, V>(a.x + (row0 + r0 + j) * a.xs + c0);
      if (a.dy) gv[j] = load_pack<E, V>(a.dy + (row0 + r0 + j) * a.dys + c0);
    }
  }
  const uint32_t call = a.call[0];
  if (blockIdx.x == 0 && threadIdx.x == 0) a.call[1] = call_after(call);  // nothing looks at that one in this kernel
  fetch_marks<T>(a, row0, call, marks);
  // The first start and the last end among the lane's rows: what belongs to them is asked for before the gates are computed.
  int first = R, last = -1;
#pragma unroll
  for (int j = R - 1; j >= 0; j--) first = marks[2 * (r0 + j)] ? j : first;
#pragma unroll
  for (int j = 0; j < R; j++) last = marks[2 * (r0 + j) + 1] ? j : last;
  float start[V], finish[V];
  load_row(a.h0, first < R ? (int64_t)(marks[2 * (r0 + first)] - 1) * a.h0s + c0 : 0, first < R && on, start);
  load_row(a.dlast, last >= 0 ? (int64_t)(marks[2 * (r0 + last) + 1] - 1) * a.dim + c0 : 0, last >= 0 && on, finish);
  float q[R][V], A[V], H[V], B[V], G[V];
#pragma unroll
  for (int j = 0; j < R; j++)
#pragma unroll
    for (int v = 0; v < V; v++) q[j][v] = gate((float)uv[j].e[v]);
#pragma unroll
  for (int v = 0; v < V; v++) { A[v] = B[v] = 1.0f; H[v] = G[v] = 0.0f; }
#pragma unroll
  for (int j = 0; j < R; j++) {
    const int32_t bag = marks[2 * (r0 + j)];
    if (bag) {
      float h0[V];
      if (j != first) load_row(a.h0, (int64_t)(bag - 1) * a.h0s + c0, on, h0);
#pragma unroll
      for (int v = 0; v < V; v++) {
        A[v] = kReset;
        H[v] = j != first ? h0[v] : start[v];
      }
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
      const float f = keep_of(q[j][v]), x = (float)xv[j].e[v];
      H[v] = f * H[v] + (a.coupled ? take_of(q[j][v]) * x : x);
      A[v] *= f;
    }
  }
#pragma unroll
  for (int j = R - 1; j >= 0; j--) {
    const int32_t ended = marks[2 * (r0 + j) + 1];
    if (ended) {
      float dl[V];
      if (j != last) load_row(a.dlast, (int64_t)(ended - 1) * a.dim + c0, on, dl);
#pragma unroll
      for (int v = 0; v < V; v++) {
        B[v] = kReset;
        G[v] = j != last ? dl[v] : finish[v];
      }
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
      opaque(q[j][v]);  // gates are unpacked anew for each pass: kept, they take half the registers
      const float f = keep_of(q[j][v]);
      G[v] = f * (G[v] + (float)gv[j].e[v]);
      B[v] *= f;
    }
  }
  bool reset = first < R, reset_back = last >= 0;
  scan_wave<V, false>(A, H, reset, a.L);
  tell_wave<V, false>(A, H, a.L, lds);
  scan_wave<V, true>(B, G, reset_back, a.L);
  tell_wave<V, true>(B, G, a.L, back);
  __syncthreads();
  for (int c = threadIdx.x; c < C; c += T) {
    const int d = tile * C + c;
    float s = 0.0f, g = 0.0f;
    if (a.chunks > 1 && d < a.dim) {
      s = a.before[(int64_t)chunk * a.dim + d];
      if (a.chained) {
        float A1, H1;
        map_of_waves<true, W>(back, C, c, A1, H1);
        g = hear_and_say<true>(a, chunk, d, call, A1, H1);
      } else {
        g = a.behind[(int64_t)chunk * a.dim + d];
      }
    }
    join_waves<false, W>(lds, C, c, s);
    join_waves<true, W>(back, C, c, g);
  }
  __syncthreads();
  float w[R][V], s[V];  // w: du / g
  start_of_lane<V, false>(A, H, reset, a.L, lds, s);
#pragma unroll
  for (int j = 0; j < R; j++) {
    const int32_t bag = marks[2 * (r0 + j)];
    if (bag) load_row(a.h0, (int64_t)(bag - 1) * a.h0s + c0, on, s);  // again: kept from above, it would take registers
#pragma unroll
    for (int v = 0; v < V; v++) {
      opaque(q[j][v]);
      const float x = (float)xv[j].e[v], f = keep_of(q[j][v]), i = take_of(q[j][v]);
      w[j][v] = (f * i) * (a.coupled ? s[v] - x : s[v]);
      s[v] = f * s[v] + (a.coupled ? i * x : x);
    }
  }
  start_of_lane<V, true>(B, G, reset_back, a.L, back, s);
  if (!on) return;
#pragma unroll
  for (int j = R - 1; j >= 0; j--) {
    const int32_t bag = marks[2 * (r0 + j)], ended = marks[2 * (r0 + j) + 1];
    if (ended) load_row(a.dlast, (int64_t)(ended - 1) * a.dim + c0, on, s);
    Pack<E, V> dx, du;
#pragma unroll
    for (int v = 0; v < V; v++) {
      opaque(q[j][v]);
      const float f = keep_of(q[j][v]), i = take_of(q[j][v]), g = (float)gv[j].e[v] + s[v];
      dx.e[v] = (E)(a.coupled ? i * g : g);
      du.e[v] = (E)(g * w[j][v]);
      s[v] = f * g;
    }
    if (r0 + j < rows) {
      store_pack<E, V>(a.dx + (row0 + r0 + j) * a.dxs + c0, dx);
      store_pack<E, V>(a.du + (row0 + r0 + j) * a.dus + c0, du);
    }
    if (bag && a.dh0)
#pragma unroll
      for (int v = 0; v < V; v++) a.dh0[(int64_t)(bag - 1) * a.dim + c0 + v] = s[v];
  }
}

// One row for each of many states, a lane an element, from element `first` on: 2 us for 7 rows of 64; what counts is the call.
template <int DT>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(int64_t first, float *state, int64_t ss, int64_t slots, const int64_t *slot_of, const typename Elem<DT>::type *x,
                                                             int64_t xs, const typename Elem<DT>::type *u, int64_t us, int64_t rows, int dim,
                                                             bool coupled, typename Elem<DT>::type *y, int64_t ys, int32_t *err) {
  const int64_t id = first + (int64_t)blockIdx.x * kThreads + threadIdx.x, r = id / dim;
  const int d = (int)(id % dim);
  if (r >= rows) return;
  const int64_t slot = slot_of ? slot_of[r] : r;
  if (slot >= slots) *err = 2;
  float h = 0.0f;
  if (slot >= 0 && slot < slots) {
    const float q = gate((float)u[r * us + d]);
    h = keep_of(q) * state[slot * ss + d] + (coupled ? take_of(q) : 1.0f) * (float)x[r * xs + d];
    state[slot * ss + d] = h;
  }
  if (y) y[r * ys + d] = (typename Elem<DT>::type)h;
}

}  // namespace

struct tbe_scan_t : DenseBase {
  int dim = 0, dtype = 0;
  bool coupled = false;
  int64_t max_bags = 0, max_rows = 0;
  Cut cut{};
  int32_t *err = nullptr;    // device: 1 = bad offsets, 2 = slot out of range
  float *maps = nullptr;     // device [chunks][2][dim]
  float *states = nullptr;   // device [chunks][dim]: before the chunks where the caller saves none, behind them in the backward
  ulonglong2 *marks = nullptr; // device [rows]
  uint32_t *call = nullptr;  // device [2]
  uint64_t *words = nullptr; // device [chunks][2][dim]
};

namespace {

int check_batch(tbe_scan_t *s, const void *x, int64_t xs, const void *u, int64_t us, const int64_t *off, int64_t bags, int64_t rows, const float *h0,
                int64_t h0s) noexcept {
  if (int rc = check_handle(s)) return rc;
  if (bags < 0 || rows < 0) return report(TBE_EINVAL, "negative number of bags or rows");
  if (bags > s->max_bags || rows > s->max_rows) return report(TBE_ELIMIT, "more bags or rows than the handle was created for");
  if (bags == 0 && rows > 0) return report(TBE_EINVAL, "rows without a bag");
  if (bags > 0 && !off) return report(TBE_EINVAL, "null offsets");
  if (rows > 0 && (!x || !u)) return report(TBE_EINVAL, "null rows or gates");
  if (xs < s->dim || us < s->dim) return report(TBE_EINVAL, "a stride below dim");
  if (h0 && h0s != 0 && h0s < s->dim) return report(TBE_EINVAL, "a stride of d_h0 that is neither 0 nor dim or more");
  return TBE_OK;
}

int64_t chunks_of(const tbe_scan_t *s, int64_t rows) { return (rows + s->cut.rows - 1) / s->cut.rows; }

template <int DT, int V>
int run(const tbe_scan_t *s, const Rows<DT> &a, bool grad, hipStream_t stream) noexcept {
  const dim3 grid((unsigned)(a.chunks * a.tiles)), joins((unsigned)((a.dim + kJoinChannels - 1) / kJoinChannels));
  const size_t tot = (size_t)2 * a.L * V * sizeof(float),  // of a wavefront
       marks = (size_t)a.chunk_rows * 2 * sizeof(int32_t);
  scan_prepare_kernel<<<dim3((unsigned)((a.bags + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(
      a.off, a.bags, a.rows, s->marks, s->call, a.dim, grad ? a.dlast : a.h0, grad ? a.dim : a.h0s, grad ? a.dh0 : a.last, s->err);
  if (a.rows == 0) return check_launch();
  const bool joined = a.chunks > 1 && !a.chained;
  if (!grad) {
    if (joined) {
      scan_sum_kernel<DT, V, false><<<grid, kThreads, kWaves * tot + marks, stream>>>(a);
      scan_join_kernel<false><<<joins, kJoinChannels * kJoinSegments, 0, stream>>>(a.maps, a.before, a.chunks, a.dim);
    }
    scan_apply_kernel<DT, V><<<grid, apply_threads(V), apply_threads(V) / 64 * tot + marks, stream>>>(a);
  } else {
    if (joined) {
      scan_sum_kernel<DT, V, true><<<grid, kThreads, kWaves * tot + marks, stream>>>(a);
      scan_join_kernel<true><<<joins, kJoinChannels * kJoinSegments, 0, stream>>>(a.maps, a.behind, a.chunks, a.dim);
    }
    scan_grad_kernel<DT, V><<<grid, grad_threads(V), grad_threads(V) / 64 * 2 * tot + marks, stream>>>(a);
  }
  return check_launch();
}

template <int DT>
int run_type(const tbe_scan_t *s, const Rows<DT> &a, bool grad, hipStream_t stream) noexcept {
  if constexpr (DT != TBE_FP32)
    if (s->cut.V == 8) return run<DT, 8>(s, a, grad, stream);
  if (s->cut.V == 4) return run<DT, 4>(s, a, grad, stream);
  return s->cut.V == 2 ? run<DT, 2>(s, a, grad, stream) : run<DT, 1>(s, a, grad, stream);
}

template <int DT>
Rows<DT> rows_of(const tbe_scan_t *s, const void *x, int64_t xs, const void *u, int64_t us, const int64_t *off, int64_t bags, int64_t rows,
                 const float *h0, int64_t h0s) {
  using E = typename Elem<DT>::type;
  Rows<DT> a = {};
  a.x = (const E *)x;
  a.u = (const E *)u;
  a.xs = xs;
  a.us = us;
  a.off = off;
  a.bags = bags;
  a.rows = rows;
  a.h0 = h0;
  a.h0s = h0s;
  a.maps = s->maps;
  a.marks = s->marks;
  a.words = s->words;
  a.call = s->call;
  a.dim = s->dim;
  a.L = s->cut.L;
  a.tiles = s->cut.tiles;
  a.chunk_rows = s->cut.rows;
  a.chunks = (int)chunks_of(s, rows);
  a.coupled = s->coupled;
  // With bags of many chunks a chunk goes through long chains of others.  262144 rows, forward and backward in us, chunks that hear / sum and
  // join: rows of 128 in bfloat16 (chunks of 64), bags of 64 rows 51 + 126 / 98 + 161, 512: 59 + 139 / 97 + 160, 2048: 86 + 187 / 97 + 160,
  // 65536: 491 + 665 / 97 + 159; of 64 in fp32 (chunks of 128), 128: 39 + 79 / 68 + 101, 2048: 48 + 91 / 68 + 100, 65536: 188 + 267 / 68 + 99.
  a.chained = rows <= bags * kChainedBags * s->cut.rows;
  return a;
}

template <int DT>
int forward(const tbe_scan_t *s, Rows<DT> a, void *y, int64_t ys, float *last, float *saved, hipStream_t stream) noexcept {
  a.y = (typename Elem<DT>::type *)y;
  a.ys = ys;
  a.last = last;
  a.before = saved ? saved : a.chained ? nullptr : s->states;
  return run_type<DT>(s, a, false, stream);
}

template <int DT>
int backward(const tbe_scan_t *s, Rows<DT> a, const float *saved, const void *dy, int64_t dys, const float *dlast, void *dx, int64_t dxs, void *du,
             int64_t dus, float *dh0, hipStream_t stream) noexcept {
  using E = typename Elem<DT>::type;
  a.before = const_cast<float *>(saved);
  a.behind = s->states;
  a.dy = (const E *)dy;
  a.dys = dys;
  a.dlast = dlast;
  a.dx = (E *)dx;
  a.dxs = dxs;
  a.du = (E *)du;
  a.dus = dus;
  a.dh0 = dh0;
  return run_type<DT>(s, a, true, stream);
}

}  // namespace

extern "C" {

int tbe_scan_create(tbe_scan_handle *out, int32_t dim, int32_t dtype, int32_t coupled, int64_t max_bags, int64_t max_rows) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (dim < 1 || dim > 65536) return report(TBE_EINVAL, "dim outside 1 .. 65536");
  if (!known_dtype(dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (max_bags < 0 || max_rows < 0) return report(TBE_EINVAL, "negative number of bags or rows");
  if (max_bags > (1ll << 38) / dim || max_rows > (1ll << 38) / dim || max_bags >= INT32_MAX)
    return report(TBE_ELIMIT, "more than 2^38 elements, or 2^31 bags");
  tbe_scan_t *s = new (std::nothrow) tbe_scan_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->dim = dim;
  s->dtype = dtype;
  s->coupled = coupled != 0;
  s->max_bags = max_bags;
  s->max_rows = max_rows;
  s->cut = cut_of(dim, dtype);
  const int64_t chunks = chunks_of(s, max_rows);
  if (chunks * s->cut.tiles > INT32_MAX / kThreads) {  // the most that a launch of the forward has, with up to 512 lanes a workgroup
    delete s;
    return report(TBE_ELIMIT, "more rows than one launch can take");
  }
  // one block: [err, call][marks][words][maps][states]
  const size_t mark_bytes = (size_t)max_rows * sizeof(ulonglong2), floats = (size_t)chunks * dim, zeros = 256 + mark_bytes + floats * 4 * sizeof(float);
  const uint32_t first_call = TBE_FIRST_CALL;  // zeros are of no call
  char *block = nullptr;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&block, zeros + floats * 3 * sizeof(float));
  if (e == hipSuccess) e = hipMemset(block, 0, zeros);
  if (e == hipSuccess) e = hipMemcpy(block + 132, &first_call, sizeof first_call, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipFree(block);
    delete s;
    return report_hip(e);
  }
  s->err = (int32_t *)block;
  s->marks = (ulonglong2 *)(block + 256);
  s->call = (uint32_t *)(block + 128);
  s->words = (uint64_t *)(block + 256 + mark_bytes);
  s->maps = (float *)(s->words + floats * 2);
  s->states = s->maps + floats * 2;
  *out = s;
  return TBE_OK;
}

int tbe_scan_destroy(tbe_scan_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->err);
  delete s;
  return TBE_OK;
}

int64_t tbe_scan_saved_floats(tbe_scan_handle s, int64_t rows) {
  if (!s || rows < 0) return report(TBE_EINVAL, "null handle or a negative number of rows");
  return chunks_of(s, rows) * s->dim;
}

int tbe_scan_forward(tbe_scan_handle s, const void *d_x, int64_t x_stride, const void *d_u, int64_t u_stride, const int64_t *d_offsets, int64_t bags,
                     int64_t rows, const float *d_h0, int64_t h0_stride, void *d_y, int64_t y_stride, float *d_last, float *d_saved,
                     void *stream) {
  if (int rc = check_batch(s, d_x, x_stride, d_u, u_stride, d_offsets, bags, rows, d_h0, h0_stride)) return rc;
  if (d_y && y_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  if (rows > 0 && d_y && (d_y == d_x || d_y == d_u)) return report(TBE_EINVAL, "the output is one of the inputs");
  if (bags == 0) return TBE_OK;
  hipStream_t st = (hipStream_t)stream;
#define ROWS(DT) rows_of<DT>(s, d_x, x_stride, d_u, u_stride, d_offsets, bags, rows, d_h0, h0_stride)
  if (s->dtype == TBE_FP32) return forward<TBE_FP32>(s, ROWS(TBE_FP32), d_y, y_stride, d_last, d_saved, st);
  if (s->dtype == TBE_FP16) return forward<TBE_FP16>(s, ROWS(TBE_FP16), d_y, y_stride, d_last, d_saved, st);
  return forward<TBE_BF16>(s, ROWS(TBE_BF16), d_y, y_stride, d_last, d_saved, st);
}

int tbe_scan_backward(tbe_scan_handle s, const void *d_x, int64_t x_stride, const void *d_u, int64_t u_stride, const int64_t *d_offsets, int64_t bags,
                      int64_t rows, const float *d_h0, int64_t h0_stride, const float *d_saved, const void *d_dy, int64_t dy_stride,
                      const float *d_dlast, void *d_dx, int64_t dx_stride, void *d_du, int64_t du_stride, float *d_dh0,
                      void *stream) {
  if (int rc = check_batch(s, d_x, x_stride, d_u, u_stride, d_offsets, bags, rows, d_h0, h0_stride)) return rc;
  if (rows > 0 && (!d_saved || !d_dx || !d_du)) return report(TBE_EINVAL, "null pointer for what the forward saved or for a gradient");
  if ((d_dy && dy_stride < s->dim) || dx_stride < s->dim || du_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  for (const void *in : {d_x, d_u, d_dy})
    if (rows > 0 && in && (d_dx == in || d_du == in)) return report(TBE_EINVAL, "an output is one of the inputs");
  if (chunks_of(s, rows) * s->cut.tiles > most_groups(grad_threads(s->cut.V))) return report(TBE_ELIMIT, "more rows than one launch can take");
  if (bags == 0) return TBE_OK;
  hipStream_t st = (hipStream_t)stream;
#define BACKWARD(DT) backward<DT>(s, ROWS(DT), d_saved, d_dy, dy_stride, d_dlast, d_dx, dx_stride, d_du, du_stride, d_dh0, st)
  if (s->dtype == TBE_FP32) return BACKWARD(TBE_FP32);
  if (s->dtype == TBE_FP16) return BACKWARD(TBE_FP16);
  return BACKWARD(TBE_BF16);
#undef BACKWARD
#undef ROWS
}

int tbe_scan_step(tbe_scan_handle s, float *d_state, int64_t state_stride, int64_t slots, const int64_t *d_slots, const void *d_x, int64_t x_stride,
                  const void *d_u, int64_t u_stride, int64_t rows, void *d_y, int64_t y_stride, void *stream) {
  if (int rc = check_handle(s)) return rc;
  if (rows < 0 || slots < 0) return report(TBE_EINVAL, "negative number of rows or slots");
  if (rows > (1ll << 38) / s->dim) return report(TBE_ELIMIT, "more than 2^38 elements");
  if (rows == 0) return TBE_OK;
  if (!d_state || !d_x || !d_u) return report(TBE_EINVAL, "null states, rows or gates");
  if (!d_slots && rows > slots) return report(TBE_EINVAL, "more rows than states");
  if (state_stride < s->dim || x_stride < s->dim || u_stride < s->dim || (d_y && y_stride < s->dim)) return report(TBE_EINVAL, "a stride below dim");
  const int64_t groups = (rows * s->dim + kThreads - 1) / kThreads;
#define LAUNCH(DT)                                                                                                                            \
  scan_step_kernel<DT><<<grid, kThreads, 0, (hipStream_t)stream>>>(done * kThreads, d_state, state_stride, slots, d_slots, (const Elem<DT>::type *)d_x, \
                                                         x_stride, (const Elem<DT>::type *)d_u, u_stride, rows, s->dim, s->coupled, (Elem<DT>::type *)d_y, y_stride, s->err)
  for (int64_t done = 0; done < groups; done += most_groups(kThreads)) {  // one launch, unless the rows have 2^32 elements
    const dim3 grid((unsigned)std::min(groups - done, most_groups(kThreads)));
    if (s->dtype == TBE_FP32) LAUNCH(TBE_FP32);
    else if (s->dtype == TBE_FP16) LAUNCH(TBE_FP16);
    else LAUNCH(TBE_BF16);
  }
#undef LAUNCH
  return check_launch();
}

int tbe_scan_check(tbe_scan_handle s, void *stream) {
  if (int rc = check_handle(s)) return rc;
  int32_t err = 0;
  hipError_t e = hipMemcpyAsync(&err, s->err, sizeof err, hipMemcpyDeviceToHost, (hipStream_t)stream);
  if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
  if (e == hipSuccess && err) {
    e = hipMemsetAsync(s->err, 0, sizeof err, (hipStream_t)stream);
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
  }
  if (e != hipSuccess) return report_hip(e);
  if (err == 1) return report(TBE_EINVAL, "offsets that do not ascend from 0 to the number of rows");
  if (err == 2) return report(TBE_ERANGE, "a slot is not below the number of states");
  return TBE_OK;
}

}  // extern "C"
