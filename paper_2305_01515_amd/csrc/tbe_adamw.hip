// AdamW over many tensors in one launch, states in 32 or 8 bits.  Contract: include/tbe.h.
// The arithmetic is written operation by operation, each rounded to fp32 (no contraction), so that a plain form in fp32
// gives the same bits: with states in 8 bits a last bit that differs now and then makes another code.
#include <cmath>
#include <new>

#include "tbe_dense.h"

using namespace tbe;

namespace {

constexpr int kThreads = 256;
constexpr int kWaveBlocks = 4;                                  // blocks of TBE_ADAMW_BLOCK elements of a workgroup: one a wavefront
constexpr int kChunk = kWaveBlocks * TBE_ADAMW_BLOCK;
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

__host__ __device__ inline uint32_t mix(uint32_t x) {  // multiplications by odd words (fractions of the roots of 2 and 3)
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

__device__ inline float load(const void *p, int dtype, int64_t i) {
  if (dtype == TBE_FP32) return ((const float *)p)[i];
  if (dtype == TBE_FP16) return (float)((const _Float16 *)p)[i];
  return (float)((const __bf16 *)p)[i];
}
__device__ inline void store(void *p, int dtype, int64_t i, float v) {
  if (dtype == TBE_FP32) ((float *)p)[i] = v;
  else if (dtype == TBE_FP16) ((_Float16 *)p)[i] = (_Float16)v;
  else ((__bf16 *)p)[i] = (__bf16)v;
}

__device__ inline float from_code(uint32_t c) {  // E4M3
  const uint32_t e = (c >> 3) & 15u, m = c & 7u;
  const float v = e ? __uint_as_float((e + 120u) << 23 | m << 20) : (float)m * 0x1p-9f;
  return c & 128u ? -v : v;
}
__device__ inline uint32_t to_code(float q, uint32_t random) {  // 0 <= q <= 448
#pragma clang fp contract(off)
  if (q < 0x1p-6f) return (uint32_t)floorf(q * 512.0f + (float)random * (1.0f / 65536.0f));
  return min(((__float_as_uint(q) + (random << 4)) >> 20) - 960u, 126u);
}

// the largest magnitude of a wavefront; a NaN is larger than an infinity, and that than any number
__device__ inline uint32_t wave_top(uint32_t bits) {
  for (int k = 32; k; k >>= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, k));
  return bits;
}

template <bool EIGHT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Tensor *tensors, const int64_t *chunk_of, int first_tensor, Grads grads, Step st,
                                                         const float *grad_scale) {
#pragma clang fp contract(off)
  const int64_t word = chunk_of[blockIdx.x];
  const int t = (int)(word >> 40);
  const void *gp = grads.p[t - first_tensor];
  if (!gp) return;
  const Tensor ts = tensors[t];
  const int lane = threadIdx.x & 63;
  const int64_t block = (word & ((1ll << 40) - 1)) * kWaveBlocks + (threadIdx.x >> 6);
  if (block * TBE_ADAMW_BLOCK >= ts.numel) return;
  const float keep = (float)(1.0 - st.lr * ts.weight_decay), gs = grad_scale ? *grad_scale : 1.0f;
  const uint32_t key = mix(st.key ^ (uint32_t)t);
  float m[4], r[4], v[4], ms = 0.0f, vs = 0.0f;
  if (EIGHT) { ms = ts.m_scale[block]; vs = ts.v_scale[block]; }
  uint32_t m_top = 0, v_top = 0;
  for (int k = 0; k < 4; k++) {
    const int64_t i = block * TBE_ADAMW_BLOCK + k * 64 + lane;
    m[k] = r[k] = v[k] = 0.0f;
    if (i >= ts.numel) continue;
    float g = load(gp, ts.grad_dtype, i);
    if (grad_scale) g = g * gs;
    float w = ts.master ? ts.master[i] : load(ts.param, ts.param_dtype, i);
    if (EIGHT) {
      m[k] = from_code(((const uint8_t *)ts.m)[i]) * ms;
      const float old = from_code(((const uint8_t *)ts.v)[i]) * vs;
      v[k] = old * old;
    } else {
      m[k] = ((const float *)ts.m)[i];
      v[k] = ((const float *)ts.v)[i];
    }
    m[k] = m[k] * st.beta1 + g * st.one_minus_beta1;
    v[k] = v[k] * st.beta2 + (g * g) * st.one_minus_beta2;
    r[k] = sqrtf(v[k]);
    w = w * keep - (m[k] * st.rate) / (r[k] * st.root + st.eps);
    if (ts.master) ts.master[i] = w;
    store(ts.param, ts.param_dtype, i, w);
    if (!EIGHT) {
      ((float *)ts.m)[i] = m[k];
      ((float *)ts.v)[i] = v[k];
    }
    m_top = max(m_top, __float_as_uint(fabsf(m[k])));
    v_top = max(v_top, __float_as_uint(fabsf(r[k])));
  }
  if (!EIGHT) return;
  const float mt = __uint_as_float(wave_top(m_top)), vt = __uint_as_float(wave_top(v_top));
  const bool mu = mt > 0.0f && mt < INFINITY, vu = vt > 0.0f && vt < INFINITY;
  const float mi = (1.0f / mt) * 448.0f, vi = (1.0f / vt) * 448.0f;
  for (int k = 0; k < 4; k++) {
    const int64_t i = block * TBE_ADAMW_BLOCK + k * 64 + lane;
    if (i >= ts.numel) continue;
    const uint32_t random = mix((uint32_t)i * 0x9E3779B9u + key);
    uint32_t mc = 0, vc = 0;
    if (mu) mc = to_code(fminf(fabsf(m[k]) * mi, 448.0f), random >> 16) + (m[k] < 0.0f ? 128u : 0u);
    if (vu && r[k] > 0.0f) vc = max(to_code(fminf(r[k] * vi, 448.0f), random & 0xFFFFu), 1u);
    ((uint8_t *)ts.m)[i] = (uint8_t)mc;
    ((uint8_t *)ts.v)[i] = (uint8_t)vc;
  }
  if (lane == 0) {
    ts.m_scale[block] = mt * (1.0f / 448.0f);
    ts.v_scale[block] = vt * (1.0f / 448.0f);
  }
}

}  // namespace

struct tbe_adamw_t : DenseBase {
  int bits = 32, n = 0;
  Tensor *tensors = nullptr;   // device [n]
  int64_t *chunk_of = nullptr; // device: tensor << 40 | chunk of it, for every workgroup
  int64_t *first = nullptr;    // host [n + 1]: first workgroup of a tensor
};

extern "C" {

int tbe_adamw_destroy(tbe_adamw_handle s) {
  if (!s) return TBE_OK;
  (void)hipFree(s->tensors);
  (void)hipFree(s->chunk_of);
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
  if (chunks > INT32_MAX) return report(TBE_ELIMIT, "more elements than one launch can take");
  tbe_adamw_t *s = new (std::nothrow) tbe_adamw_t;
  Tensor *host = new (std::nothrow) Tensor[num_tensors];
  int64_t *chunk_of = new (std::nothrow) int64_t[chunks + 1];
  int rc = TBE_OK;
  if (s) s->first = new (std::nothrow) int64_t[num_tensors + 1];
  if (!s || !host || !chunk_of || !s->first) {
    rc = report(TBE_ENOMEM, "no memory for the handle");
  } else {
    s->bits = state_bits;
    s->n = num_tensors;
      int64_t at = 0;
    for (int t = 0; t < num_tensors; t++) {
      const tbe_adamw_tensor &a = h_tensors[t];
      host[t] = {a.d_param, a.d_master, a.d_m, a.d_v, a.d_m_scale, a.d_v_scale, a.numel, a.weight_decay, a.param_dtype, a.grad_dtype};
      s->first[t] = at;
      for (int64_t c = 0; c < (a.numel + kChunk - 1) / kChunk; c++) chunk_of[at++] = (int64_t)t << 40 | c;
    }
    s->first[num_tensors] = at;
    hipError_t e = hipGetDevice(&s->device);
    if (e == hipSuccess) e = hipMalloc((void **)&s->tensors, num_tensors * sizeof(Tensor));
    if (e == hipSuccess) e = hipMalloc((void **)&s->chunk_of, (chunks + 1) * sizeof(int64_t));
    if (e == hipSuccess) e = hipMemcpy(s->tensors, host, num_tensors * sizeof(Tensor), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(s->chunk_of, chunk_of, chunks * sizeof(int64_t), hipMemcpyHostToDevice);
    if (e != hipSuccess) rc = report_hip(e);
  }
  delete[] host;
  delete[] chunk_of;
  if (rc) {
    (void)tbe_adamw_destroy(s);
    return rc;
  }
  *out = s;
  return TBE_OK;
}

int tbe_adamw_step(tbe_adamw_handle s, const void *const *h_grads, int64_t step, double lr, double beta1, double beta2, double eps, uint32_t seed,
                   const float *d_grad_scale, void *stream) {
  if (int rc = check_handle(s)) return rc;
  if (!h_grads) return report(TBE_EINVAL, "null gradients");
  if (step < 1) return report(TBE_EINVAL, "the first step is step 1");
  if (!(lr >= 0.0) || !std::isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps))
    return report(TBE_EINVAL, "lr and eps are at least 0, the betas at least 0 and below 1");
  Step st;
  st.beta1 = (float)beta1;
  st.one_minus_beta1 = (float)(1.0 - beta1);
  st.beta2 = (float)beta2;
  st.one_minus_beta2 = (float)(1.0 - beta2);
  st.rate = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  st.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  st.eps = (float)eps;
  st.lr = lr;
  st.key = mix(mix(seed) ^ (uint32_t)step);
  for (int t0 = 0; t0 < s->n; t0 += kMaxGrads) {
    const int t1 = t0 + kMaxGrads < s->n ? t0 + kMaxGrads : s->n;
    const int64_t first = s->first[t0], count = s->first[t1] - first;
    if (count == 0) continue;
    Grads g = {};
    for (int t = t0; t < t1; t++) g.p[t - t0] = h_grads[t];
    if (s->bits == 8) adamw_kernel<true><<<dim3((unsigned)count), kThreads, 0, (hipStream_t)stream>>>(s->tensors, s->chunk_of + first, t0, g, st, d_grad_scale);
    else adamw_kernel<false><<<dim3((unsigned)count), kThreads, 0, (hipStream_t)stream>>>(s->tensors, s->chunk_of + first, t0, g, st, d_grad_scale);
  }
  return check_launch();
}

}  // extern "C"
