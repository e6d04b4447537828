// AdamW over many tensors in one launch, states in 32 or 8 bits.  Contract: include/tbe.h.
//
// Bound by memory: 28 bytes an element with fp32 everywhere, 16 with states in 8 bits (fp32 weights and gradients, or 16-bit ones with an
// fp32 copy).  172 M weights: 880 us (5.5 TB/s) and 503 to 532 us by card (5.2 to 5.5 TB/s).  A wavefront has a block of TBE_ADAMW_BLOCK elements, 4 side by
// side a lane, so that the largest of a block is an exchange between lanes and every load is 4 elements of its type.  (Two blocks a
// wavefront took 4 % longer with fp32 states, 1.5 % in 8 bits.)  The types are the tensor's: one kernel has a body for
// each combination and takes the one that its workgroup's tensor asks for.
//
// Moving averages and their codes are computed operation by operation, each rounded to fp32 (no contraction), so that a plain form in fp32
// gives the same bits: a last bit that differs makes another code now and then, and a code is a sixteenth of its value.
#include <algorithm>
#include <cmath>
#include <new>

#include "tbe_dense.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = kThreads / 64 * TBE_ADAMW_BLOCK;          // elements of a workgroup: a block for each wavefront
constexpr int kMaxGrads = 256;                                  // tensors of a launch: their gradients' addresses are kernel arguments

struct Tensor {
  void *param;
  float *master;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t numel;
  double weight_decay;
  int32_t param_dtype, grad_dtype;
};

struct Grads {
  const void *p[kMaxGrads];
};

struct Step {
  float beta1, one_minus_beta1, beta2, one_minus_beta2, rate, root, eps;
  double lr;
  uint32_t key;  // of seed and step
};

// What of a Step goes by its number, where that is in device memory
struct Counted {
  float rate, root;
  uint32_t key;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {  // multiplications by odd words (fractions of the roots of 2 and 3)
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

__host__ __device__ inline Counted counted_of(int64_t step, double lr, double beta1, double beta2, uint32_t seed) {
  return {(float)(lr / (1.0 - pow(beta1, (double)step))), (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step))), mix(mix(seed) ^ (uint32_t)step)};
}

// A lane in front of a step that is counted on the GPU: 2 us.  (One in the step's own kernel would have to wait for all of it, or count in each workgroup.)
__global__ void adamw_count_kernel(int64_t *step, double lr, double beta1, double beta2, uint32_t seed, Counted *out) {
  const int64_t n = max(*step + 1, (int64_t)1);
  *step = n;
  *out = counted_of(n, lr, beta1, beta2, seed);
}

// Addresses that come out of memory: told to be of device memory, or the compiler takes instructions that look for LDS as well.
template <class T>
__device__ inline T *global(T *p) { return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p; }

// 4 elements side by side, at any address that an element may have; `n` of them where the tensor ends
template <int DT>
__device__ inline Pack<typename Elem<DT>::type, 4> load4(const void *p, int64_t i, int n) {
  using E = typename Elem<DT>::type;
  Pack<E, 4> r = {};
  if (n >= 4) __builtin_memcpy(&r, (const E *)p + i, sizeof r);
  else
#pragma unroll
    for (int k = 0; k < 3; k++)
      if (k < n) r.e[k] = ((const E *)p)[i + k];
  return r;
}
template <int DT>
__device__ inline void store4(void *p, int64_t i, int n, const float (&v)[4]) {
  using E = typename Elem<DT>::type;
  Pack<E, 4> r;
#pragma unroll
  for (int k = 0; k < 4; k++) r.e[k] = (E)v[k];
  if (n >= 4) __builtin_memcpy((E *)p + i, &r, sizeof r);
  else
#pragma unroll
    for (int k = 0; k < 3; k++)
      if (k < n) ((E *)p)[i + k] = r.e[k];
}
__device__ inline uint32_t load_codes(const void *p, int64_t i, int n) {
  uint32_t r = 0;
  if (n >= 4) __builtin_memcpy(&r, (const uint8_t *)p + i, 4);
  else
#pragma unroll
    for (int k = 0; k < 3; k++)
      if (k < n) r |= (uint32_t)((const uint8_t *)p)[i + k] << (8 * k);
  return r;
}
__device__ inline void store_codes(void *p, int64_t i, int n, uint32_t c) {
  if (n >= 4) __builtin_memcpy((uint8_t *)p + i, &c, 4);
  else
#pragma unroll
    for (int k = 0; k < 3; k++)
      if (k < n) ((uint8_t *)p)[i + k] = (uint8_t)(c >> (8 * k));
}

typedef float float2v __attribute__((ext_vector_type(2)));
__device__ inline void from_codes(uint32_t c, float (&v)[4]) {  // E4M3, exact
  const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  v[0] = lo.x;
  v[1] = lo.y;
  v[2] = hi.x;
  v[3] = hi.y;
}
// 0 <= q <= 448 to a code: the upper of two where the 16 random bits, as a share of their distance, reach beyond it
__device__ inline uint32_t to_code(float q, uint32_t random) {
#pragma clang fp contract(off)
  const uint32_t normal = ((__float_as_uint(q) + (random << 4)) >> 20) - 960u;
  const uint32_t small = (uint32_t)(q * 512.0f + (float)random * (1.0f / 65536.0f));
  return min(q < 0x1p-6f ? small : normal, 126u);
}

// the largest magnitude of a wavefront; a NaN is larger than an infinity, and that than any number
__device__ inline uint32_t wave_top(uint32_t bits) {
  for (int k = 32; k; k >>= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, k));
  return bits;
}

template <bool EIGHT, int PT, int GT, bool MASTER>
__device__ inline void step_block(const Tensor &ts, const void *gp, uint32_t key, int64_t block, const Step &st, const float *grad_scale) {
#pragma clang fp contract(off)
  constexpr int WT = MASTER ? (int)TBE_FP32 : PT;  // what the weight is held in
  const int lane = threadIdx.x & 63;
  const float keep = (float)(1.0 - st.lr * ts.weight_decay), gs = grad_scale ? *grad_scale : 1.0f;
  const int64_t i = block * TBE_ADAMW_BLOCK + lane * 4;
  if (block * TBE_ADAMW_BLOCK >= ts.numel) return;  // the same in all lanes
  const int n = (int)min((int64_t)4, ts.numel - i);
  const auto g = load4<GT>(gp, i, n);
  const auto w = load4<WT>(MASTER ? (const void *)ts.master : ts.param, i, n);
  float m[4], v[4], r[4], x[4];
  if (EIGHT) {
    const uint32_t mc = load_codes(ts.m, i, n), vc = load_codes(ts.v, i, n);
    const float ms = ts.m_scale[block], vs = ts.v_scale[block];
    from_codes(mc, m);
    from_codes(vc, v);
#pragma unroll
    for (int k = 0; k < 4; k++) {
      m[k] = m[k] * ms;
      v[k] = v[k] * vs;
      v[k] = v[k] * v[k];
    }
  } else {
    const auto m32 = load4<TBE_FP32>(ts.m, i, n), v32 = load4<TBE_FP32>(ts.v, i, n);
#pragma unroll
    for (int k = 0; k < 4; k++) {
      m[k] = m32.e[k];
      v[k] = v32.e[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; k++) {
    float gk = (float)g.e[k];
    if (grad_scale) gk = gk * gs;
    m[k] = m[k] * st.beta1 + gk * st.one_minus_beta1;
    v[k] = v[k] * st.beta2 + (gk * gk) * st.one_minus_beta2;
    r[k] = sqrtf(v[k]);
    // the quotient by a reciprocal of an ulp: an error far below that of the weight it changes
    x[k] = (float)w.e[k] * keep - (m[k] * st.rate) * __builtin_amdgcn_rcpf(r[k] * st.root + st.eps);
  }
  if (MASTER) store4<TBE_FP32>(ts.master, i, n, x);
  store4<PT>(ts.param, i, n, x);
  if (!EIGHT) {
    store4<TBE_FP32>(ts.m, i, n, m);
    store4<TBE_FP32>(ts.v, i, n, v);
    return;
  }
  uint32_t m_top = 0, v_top = 0;
#pragma unroll
  for (int k = 0; k < 4; k++)
    if (k < n) {  // zeros behind the end would not count, but what a NaN grad_scale makes of them would
      m_top = max(m_top, __float_as_uint(fabsf(m[k])));
      v_top = max(v_top, __float_as_uint(r[k]));
    }
  const float mt = __uint_as_float(wave_top(m_top)), vt = __uint_as_float(wave_top(v_top));
  // 448 / mt is a number of fp32 from 2^-119 up (a root of an fp32 number is never below that): a block below is stored as zeros, its codes would
  // all be that of the largest.  (Taken times 2^64 first, 172 M weights take 526 us instead of 520.)
  const bool mu = mt >= 0x1p-119f && mt < INFINITY, vu = vt > 0.0f && vt < INFINITY;
  const float mi = (1.0f / mt) * 448.0f, vi = (1.0f / vt) * 448.0f;
  uint32_t mw = 0, vw = 0;
#pragma unroll
  for (int k = 0; k < 4; k++) {
    const uint32_t random = mix((uint32_t)(i + k) * 0x9E3779B9u + key);
    const uint32_t a = to_code(fminf(fabsf(m[k]) * mi, 448.0f), random >> 16) | (__float_as_uint(m[k]) >> 24 & 128u);
    const uint32_t c = max(to_code(fminf(r[k] * vi, 448.0f), random & 0xFFFFu), 1u);  // above zero: never zero
    mw |= (m[k] != 0.0f ? a : 0u) << (8 * k);
    vw |= (r[k] > 0.0f ? c : 0u) << (8 * k);
  }
  store_codes(ts.m, i, n, mu ? mw : 0u);
  store_codes(ts.v, i, n, vu ? vw : 0u);
  if (lane == 0) {
    ts.m_scale[block] = mt * (1.0f / 448.0f);
    ts.v_scale[block] = vt * (1.0f / 448.0f);
  }
}

template <bool EIGHT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Tensor *tensors, const int64_t *chunk_list, int first_tensor, Grads grads, Step st,
                                                         const float *grad_scale, const Counted *counted) {
  if (counted) {
    st.rate = counted->rate;
    st.root = counted->root;
    st.key = counted->key;
  }
  const int64_t word = chunk_list[blockIdx.x];
  const int t = (int)(word >> 40);
  const void *gp = global((const char *)grads.p[t - first_tensor]);
  if (!gp) return;
  Tensor ts = tensors[t];
  ts.param = global((char *)ts.param);
  ts.master = global(ts.master);
  ts.m = global((char *)ts.m);
  ts.v = global((char *)ts.v);
  ts.m_scale = global(ts.m_scale);
  ts.v_scale = global(ts.v_scale);
  const uint32_t key = mix(st.key ^ (uint32_t)t);
  const int64_t block = (word & ((1ll << 40) - 1)) * (kThreads / 64) + (threadIdx.x >> 6);
  const int kind = ts.param_dtype * 3 + ts.grad_dtype;
#define BODY(PT, GT)                                                                          \
  case PT * 3 + GT:                                                                           \
    if (ts.master) step_block<EIGHT, PT, GT, true>(ts, gp, key, block, st, grad_scale);      \
    else step_block<EIGHT, PT, GT, false>(ts, gp, key, block, st, grad_scale);               \
    return;
  switch (kind) {
    BODY(0, 0) BODY(0, 1) BODY(0, 2) BODY(1, 0) BODY(1, 1) BODY(1, 2) BODY(2, 0) BODY(2, 1) BODY(2, 2)
  }
#undef BODY
}

}  // namespace

struct tbe_adamw_t : DenseBase {
  int bits = 32, n = 0;
  Tensor *tensors = nullptr;   // device [n]
  int64_t *chunk_list = nullptr; // device: tensor << 40 | chunk of it, for every workgroup
  int64_t *first = nullptr;    // host [n + 1]: first workgroup of a tensor
  Counted *counted = nullptr;  // device
};

namespace {

// A step with the number `step`, or with that behind *d_step
int run(tbe_adamw_t *s, const void *const *h_grads, int64_t step, int64_t *d_step, double lr, double beta1, double beta2, double eps, uint32_t seed,
        const float *d_grad_scale, hipStream_t stream) noexcept {
  if (int rc = check_handle(s)) return rc;
  if (!h_grads) return report(TBE_EINVAL, "null gradients");
  if (!(lr >= 0.0) || !std::isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps))
    return report(TBE_EINVAL, "lr and eps are at least 0, the betas at least 0 and below 1");
  Step st;
  st.beta1 = (float)beta1;
  st.one_minus_beta1 = (float)(1.0 - beta1);
  st.beta2 = (float)beta2;
  st.one_minus_beta2 = (float)(1.0 - beta2);
  st.eps = (float)eps;
  st.lr = lr;
  const Counted c = counted_of(step, lr, beta1, beta2, seed);
  st.rate = c.rate;
  st.root = c.root;
  st.key = c.key;
  if (d_step) adamw_count_kernel<<<1, 1, 0, stream>>>(d_step, lr, beta1, beta2, seed, s->counted);
  const Counted *counted = d_step ? s->counted : nullptr;
  for (int t0 = 0; t0 < s->n; t0 += kMaxGrads) {
    const int t1 = t0 + kMaxGrads < s->n ? t0 + kMaxGrads : s->n;
    const int64_t first = s->first[t0], count = s->first[t1] - first;
    if (count == 0) continue;
    Grads g = {};
    for (int t = t0; t < t1; t++) g.p[t - t0] = h_grads[t];
    for (int64_t done = 0; done < count; done += most_groups(kThreads)) {  // one launch, unless the tensors have 1.7e10 elements
      const dim3 grid((unsigned)std::min(count - done, most_groups(kThreads)));
      const int64_t *list = s->chunk_list + first + done;
      if (s->bits == 8) adamw_kernel<true><<<grid, kThreads, 0, stream>>>(s->tensors, list, t0, g, st, d_grad_scale, counted);
      else adamw_kernel<false><<<grid, kThreads, 0, stream>>>(s->tensors, list, t0, g, st, d_grad_scale, counted);
    }
  }
  return check_launch();
}

}  // namespace

extern "C" {

int tbe_adamw_destroy(tbe_adamw_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->tensors);
  (void)hipFree(s->chunk_list);
  delete[] s->first;
  delete s;
  return TBE_OK;
}

int tbe_adamw_create(tbe_adamw_handle *out, const tbe_adamw_tensor *h_tensors, int32_t num_tensors, int32_t state_bits) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (!h_tensors || num_tensors < 1) return report(TBE_EINVAL, "no tensors");
  if (state_bits != 32 && state_bits != 8) return report(TBE_EINVAL, "states have 32 or 8 bits");
  if (num_tensors > 1 << 20) return report(TBE_ELIMIT, "more than 2^20 tensors");
  int64_t chunks = 0;
  for (int t = 0; t < num_tensors; t++) {
    const tbe_adamw_tensor &a = h_tensors[t];
    if (a.numel < 0) return report(TBE_EINVAL, "a tensor of negative size");
    if (a.numel > 1ll << 40) return report(TBE_ELIMIT, "a tensor of more than 2^40 elements");
    if (!known_dtype(a.param_dtype) || !known_dtype(a.grad_dtype)) return report(TBE_EINVAL, "unknown dtype");
    if (a.numel && (!a.d_param || !a.d_m || !a.d_v || (state_bits == 8 && (!a.d_m_scale || !a.d_v_scale))))
      return report(TBE_EINVAL, "null parameter or state");
    if (!std::isfinite(a.weight_decay)) return report(TBE_EINVAL, "weight_decay is not finite");
    chunks += (a.numel + kChunk - 1) / kChunk;
  }
  if (chunks > INT32_MAX) return report(TBE_ELIMIT, "more than 2^41 elements");
  tbe_adamw_t *s = new (std::nothrow) tbe_adamw_t;
  Tensor *host = new (std::nothrow) Tensor[num_tensors];
  int64_t *list = new (std::nothrow) int64_t[chunks + 1];
  int rc = TBE_OK;
  if (s) s->first = new (std::nothrow) int64_t[num_tensors + 1];
  if (!s || !host || !list || !s->first) {
    rc = report(TBE_ENOMEM, "no memory for the handle");
  } else {
    s->bits = state_bits;
    s->n = num_tensors;
      int64_t at = 0;
    for (int t = 0; t < num_tensors; t++) {
      const tbe_adamw_tensor &a = h_tensors[t];
      host[t] = {a.d_param, a.d_master, a.d_m, a.d_v, a.d_m_scale, a.d_v_scale, a.numel, a.weight_decay, a.param_dtype, a.grad_dtype};
      s->first[t] = at;
      for (int64_t c = 0; c < (a.numel + kChunk - 1) / kChunk; c++) list[at++] = (int64_t)t << 40 | c;
    }
    s->first[num_tensors] = at;
    hipError_t e = hipGetDevice(&s->device);
    if (e == hipSuccess) e = hipMalloc((void **)&s->tensors, num_tensors * sizeof(Tensor) + sizeof(Counted));  // one block: [tensors][counted]
    s->counted = (Counted *)(s->tensors + num_tensors);
    if (e == hipSuccess) e = hipMalloc((void **)&s->chunk_list, (chunks + 1) * sizeof(int64_t));
    if (e == hipSuccess) e = hipMemcpy(s->tensors, host, num_tensors * sizeof(Tensor), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(s->chunk_list, list, chunks * sizeof(int64_t), hipMemcpyHostToDevice);
    if (e != hipSuccess) rc = report_hip(e);
  }
  delete[] host;
  delete[] list;
  if (rc) {
    (void)tbe_adamw_destroy(s);
    return rc;
  }
  *out = s;
  return TBE_OK;
}

int tbe_adamw_step(tbe_adamw_handle s, const void *const *h_grads, int64_t step, double lr, double beta1, double beta2, double eps, uint32_t seed,
                   const float *d_grad_scale, void *stream) {
  if (s && step < 1) return report(TBE_EINVAL, "the first step is step 1");
  return run(s, h_grads, step, nullptr, lr, beta1, beta2, eps, seed, d_grad_scale, (hipStream_t)stream);
}

int tbe_adamw_step_counted(tbe_adamw_handle s, const void *const *h_grads, int64_t *d_step, double lr, double beta1, double beta2, double eps, uint32_t seed,
                           const float *d_grad_scale, void *stream) {
  if (s && !d_step) return report(TBE_EINVAL, "null step number");
  return run(s, h_grads, 1, d_step, lr, beta1, beta2, eps, seed, d_grad_scale, (hipStream_t)stream);
}

}  // extern "C"
