// Gated linear recurrence over the rows of every bag: forward, backward, one row for each of many states.
// Contract: include/tbe.h.
#include <cmath>
#include <new>

#include "tbe_dense.h"

using namespace tbe;

struct tbe_scan_t : DenseBase {
  int dim = 0, dtype = 0;
  bool coupled = false;
  int64_t max_bags = 0, max_rows = 0;
  int32_t *err = nullptr;  // device: 1 = bad offsets, 2 = slot out of range
};

namespace {

constexpr int kThreads = 256;

struct Gate {
  float f, i;  // 1 / (1 + exp(-u)) and one less it
};
__device__ inline Gate gate(float u) {
  const float e = __expf(-fabsf(u)), big = 1.0f / (1.0f + e), small = e * big;
  return u >= 0.0f ? Gate{big, small} : Gate{small, big};
}

// offsets ascend from 0 to rows: bags outside that are left out, and the call is reported by tbe_scan_check
__device__ inline bool bag_rows(const int64_t *off, int64_t b, int64_t rows, int64_t &lo, int64_t &hi) {
  lo = off[b];
  hi = off[b + 1];
  return lo >= 0 && lo <= hi && hi <= rows;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void scan_forward_kernel(const typename Elem<DT>::type *x, int64_t xs, const typename Elem<DT>::type *u,
                                                                int64_t us, const int64_t *off, int64_t bags, int64_t rows, int dim, bool coupled,
                                                                const float *h0, int64_t h0s, typename Elem<DT>::type *y, int64_t ys, float *last,
                                                                float *saved, int32_t *err) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = id / dim;
  const int d = (int)(id % dim);
  if (b >= bags) return;
  int64_t lo, hi;
  if ((b == 0 && off[0] != 0) || (b == bags - 1 && off[bags] != rows)) *err = 1;
  if (!bag_rows(off, b, rows, lo, hi)) { *err = 1; return; }
  float h = h0 ? h0[b * h0s + d] : 0.0f;
  for (int64_t t = lo; t < hi; t++) {
    const Gate g = gate((float)u[t * us + d]);
    h = g.f * h + (coupled ? g.i : 1.0f) * (float)x[t * xs + d];
    if (y) y[t * ys + d] = (typename Elem<DT>::type)h;
    if (saved) saved[t * dim + d] = h;
  }
  if (last) last[b * dim + d] = h;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void scan_backward_kernel(const typename Elem<DT>::type *x, int64_t xs, const typename Elem<DT>::type *u,
                                                                 int64_t us, const int64_t *off, int64_t bags, int64_t rows, int dim, bool coupled,
                                                                 const float *h0, int64_t h0s, const float *saved, const typename Elem<DT>::type *dy,
                                                                 int64_t dys, const float *dlast, typename Elem<DT>::type *dx, int64_t dxs,
                                                                 typename Elem<DT>::type *du, int64_t dus, float *dh0, int32_t *err) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = id / dim;
  const int d = (int)(id % dim);
  if (b >= bags) return;
  int64_t lo, hi;
  if ((b == 0 && off[0] != 0) || (b == bags - 1 && off[bags] != rows)) *err = 1;
  if (!bag_rows(off, b, rows, lo, hi)) { *err = 1; return; }
  float c = dlast ? dlast[b * dim + d] : 0.0f;
  for (int64_t t = hi - 1; t >= lo; t--) {
    const Gate g = gate((float)u[t * us + d]);
    const float xv = (float)x[t * xs + d], before = t > lo ? saved[(t - 1) * dim + d] : h0 ? h0[b * h0s + d] : 0.0f;
    const float gt = (dy ? (float)dy[t * dys + d] : 0.0f) + c;
    dx[t * dxs + d] = (typename Elem<DT>::type)(coupled ? g.i * gt : gt);
    du[t * dus + d] = (typename Elem<DT>::type)(gt * (coupled ? before - xv : before) * g.f * g.i);
    c = g.f * gt;
  }
  if (dh0) dh0[b * dim + d] = c;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(float *state, int64_t ss, int64_t slots, const int64_t *slot_of, const typename Elem<DT>::type *x,
                                                             int64_t xs, const typename Elem<DT>::type *u, int64_t us, int64_t rows, int dim,
                                                             bool coupled, typename Elem<DT>::type *y, int64_t ys, int32_t *err) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, r = id / dim;
  const int d = (int)(id % dim);
  if (r >= rows) return;
  const int64_t slot = slot_of ? slot_of[r] : r;
  if (slot >= slots) *err = 2;
  float h = 0.0f;
  if (slot >= 0 && slot < slots) {
    const Gate g = gate((float)u[r * us + d]);
    h = g.f * state[slot * ss + d] + (coupled ? g.i : 1.0f) * (float)x[r * xs + d];
    state[slot * ss + d] = h;
  }
  if (y) y[r * ys + d] = (typename Elem<DT>::type)h;
}

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

dim3 grid_of(int64_t n) { return dim3((unsigned)((n + kThreads - 1) / kThreads)); }

}  // namespace

extern "C" {

int tbe_scan_create(tbe_scan_handle *out, int32_t dim, int32_t dtype, int32_t coupled, int64_t max_bags, int64_t max_rows) {
  if (!out) return report(TBE_EINVAL, "null pointer for the handle");
  *out = nullptr;
  if (dim < 1 || dim > 65536) return report(TBE_EINVAL, "dim outside 1 .. 65536");
  if (!known_dtype(dtype)) return report(TBE_EINVAL, "unknown dtype");
  if (max_bags < 0 || max_rows < 0) return report(TBE_EINVAL, "negative number of bags or rows");
  if (max_bags > (1ll << 38) / dim || max_rows > (1ll << 38) / dim) return report(TBE_ELIMIT, "more than 2^38 elements");
  tbe_scan_t *s = new (std::nothrow) tbe_scan_t;
  if (!s) return report(TBE_ENOMEM, "no memory for the handle");
  s->dim = dim;
  s->dtype = dtype;
  s->coupled = coupled != 0;
  s->max_bags = max_bags;
  s->max_rows = max_rows;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc((void **)&s->err, 256);
  if (e == hipSuccess) e = hipMemset(s->err, 0, 256);
  if (e != hipSuccess) {
    (void)hipFree(s->err);
    delete s;
    return report_hip(e);
  }
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
  return rows * s->dim;
}

int tbe_scan_forward(tbe_scan_handle s, const void *d_x, int64_t x_stride, const void *d_u, int64_t u_stride, const int64_t *d_offsets, int64_t bags,
                     int64_t rows, const float *d_h0, int64_t h0_stride, void *d_y, int64_t y_stride, float *d_last, float *d_saved,
                     void *stream) {
  if (int rc = check_batch(s, d_x, x_stride, d_u, u_stride, d_offsets, bags, rows, d_h0, h0_stride)) return rc;
  if (d_y && y_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  if (bags == 0) return TBE_OK;
  const dim3 grid = grid_of(bags * s->dim);
#define LAUNCH(DT)                                                                                                                            \
  scan_forward_kernel<DT><<<grid, kThreads, 0, (hipStream_t)stream>>>((const Elem<DT>::type *)d_x, x_stride, (const Elem<DT>::type *)d_u, u_stride, d_offsets, \
                                                            bags, rows, s->dim, s->coupled, d_h0, h0_stride, (Elem<DT>::type *)d_y, y_stride, \
                                                            d_last, d_saved, s->err)
  if (s->dtype == TBE_FP32) LAUNCH(TBE_FP32);
  else if (s->dtype == TBE_FP16) LAUNCH(TBE_FP16);
  else LAUNCH(TBE_BF16);
#undef LAUNCH
  return check_launch();
}

int tbe_scan_backward(tbe_scan_handle s, const void *d_x, int64_t x_stride, const void *d_u, int64_t u_stride, const int64_t *d_offsets, int64_t bags,
                      int64_t rows, const float *d_h0, int64_t h0_stride, const float *d_saved, const void *d_dy, int64_t dy_stride,
                      const float *d_dlast, void *d_dx, int64_t dx_stride, void *d_du, int64_t du_stride, float *d_dh0,
                      void *stream) {
  if (int rc = check_batch(s, d_x, x_stride, d_u, u_stride, d_offsets, bags, rows, d_h0, h0_stride)) return rc;
  if (rows > 0 && (!d_saved || !d_dx || !d_du)) return report(TBE_EINVAL, "null pointer for what the forward saved or for a gradient");
  if ((d_dy && dy_stride < s->dim) || dx_stride < s->dim || du_stride < s->dim) return report(TBE_EINVAL, "a stride below dim");
  if (bags == 0) return TBE_OK;
  const dim3 grid = grid_of(bags * s->dim);
#define LAUNCH(DT)                                                                                                                             \
  scan_backward_kernel<DT><<<grid, kThreads, 0, (hipStream_t)stream>>>((const Elem<DT>::type *)d_x, x_stride, (const Elem<DT>::type *)d_u, u_stride, d_offsets, \
                                                             bags, rows, s->dim, s->coupled, d_h0, h0_stride, d_saved, (const Elem<DT>::type *)d_dy, \
                                                             dy_stride, d_dlast, (Elem<DT>::type *)d_dx, dx_stride, (Elem<DT>::type *)d_du, du_stride, \
                                                             d_dh0, s->err)
  if (s->dtype == TBE_FP32) LAUNCH(TBE_FP32);
  else if (s->dtype == TBE_FP16) LAUNCH(TBE_FP16);
  else LAUNCH(TBE_BF16);
#undef LAUNCH
  return check_launch();
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
  const dim3 grid = grid_of(rows * s->dim);
#define LAUNCH(DT)                                                                                                                            \
  scan_step_kernel<DT><<<grid, kThreads, 0, (hipStream_t)stream>>>(d_state, state_stride, slots, d_slots, (const Elem<DT>::type *)d_x, x_stride,        \
                                                         (const Elem<DT>::type *)d_u, u_stride, rows, s->dim, s->coupled, (Elem<DT>::type *)d_y, y_stride, s->err)
  if (s->dtype == TBE_FP32) LAUNCH(TBE_FP32);
  else if (s->dtype == TBE_FP16) LAUNCH(TBE_FP16);
  else LAUNCH(TBE_BF16);
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
