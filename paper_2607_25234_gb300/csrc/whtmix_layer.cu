// whtmix_layer.cu -- the C ABI's entry points of the layer around the mixer: RMS norm (whtmix_norm.cu), layer norm
// (whtmix_layer_norm.cu), the matrix product with its epilogue (whtmix_linear.cu), the gated feed-forward half (whtmix_gated.cu) and the
// clipping of a step's gradients (whtmix_clip.cu).  Every check runs before anything is enqueued; a failing call enqueues and writes
// nothing.
#include <cuda_runtime.h>

#include <algorithm>
#include <vector>

#include "whtmix.h"
#include "whtmix_clip.cuh"
#include "whtmix_gated.cuh"
#include "whtmix_host.cuh"
#include "whtmix_kernels.cuh"
#include "whtmix_layer_norm.cuh"
#include "whtmix_linear.cuh"
#include "whtmix_norm.cuh"

using namespace whtmix;

namespace {

constexpr int64_t MAX_CHANNELS = int64_t{1} << 24, MAX_TOKENS = (int64_t{1} << 31) - 256, MAX_ELEMENTS = int64_t{1} << 40,
                  MAX_TENSORS = int64_t{1} << 20;

// A row matrix (or, with rows = 1, a vector) of the call: its address range, for the checks of alignment and overlap.
struct Range {
  const void* p;
  int64_t rows, cols, stride;
  int es;
  size_t bytes() const { return p ? static_cast<size_t>((rows - 1) * stride + cols) * es : 0; }
  bool same(const Range& o) const { return p == o.p && (rows <= 1 || stride == o.stride) && es == o.es; }
};

bool overlap(const Range& a, const Range& b) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const size_t na = a.bytes(), nb = b.bytes();
  return na && nb && pa < pb + nb && pb < pa + na;
}

int check_sizes(int64_t T, int64_t a, int64_t b) {
  if (T < 0 || a < 1 || b < 1) return WHTMIX_ERR_INVALID_ARG;
  if (a > MAX_CHANNELS || b > MAX_CHANNELS || T > MAX_TOKENS) return WHTMIX_ERR_BAD_SHAPE;
  if (T * a > MAX_ELEMENTS || T * b > MAX_ELEMENTS || a * b > MAX_ELEMENTS) return WHTMIX_ERR_BAD_SHAPE;
  return WHTMIX_OK;
}

// Strides, alignment to the element and overlap of a call's matrices: outputs first.  free(o, i): output o may be input i itself.
template <int O, int I, class F>
int check_ranges(const Range (&out)[O], const Range (&in)[I], F&& may_be) {
  auto one = [](const Range& r) -> int {
    if (!r.p) return WHTMIX_OK;
    if (r.rows > 1 && r.stride < r.cols) return WHTMIX_ERR_INVALID_ARG;
    if (r.rows > 1 && r.stride > MAX_ELEMENTS / r.rows) return WHTMIX_ERR_BAD_SHAPE;
    return (reinterpret_cast<uintptr_t>(r.p) & (r.es - 1)) ? WHTMIX_ERR_MISALIGNED : WHTMIX_OK;
  };
  for (const Range& r : out)
    if (const int rc = one(r)) return rc;
  for (const Range& r : in)
    if (const int rc = one(r)) return rc;
  for (int o = 0; o < O; ++o) {
    for (int i = 0; i < I; ++i)
      if (overlap(out[o], in[i]) && !(may_be(o, i) && out[o].same(in[i]))) return WHTMIX_ERR_ALIAS;
    for (int q = o + 1; q < O; ++q)
      if (overlap(out[o], out[q])) return WHTMIX_ERR_ALIAS;
  }
  return WHTMIX_OK;
}

// No C++ exception leaves a C entry (the workspace cache allocates host memory).
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return host::fail(cudaErrorMemoryAllocation);
  }
}

int zero(void* p, size_t bytes, cudaStream_t stream) {
  if (!p) return WHTMIX_OK;
  const cudaError_t e = cudaMemsetAsync(p, 0, bytes, stream);
  return e == cudaSuccess ? WHTMIX_OK : host::fail(e);
}

// Slot-0 workspace of the stream: the error word that whtmix_sync reads.
int error_word(int dev, cudaStream_t stream, unsigned int** err) {
  void* ws = nullptr;
  const int rc = host::workspace(dev, stream, sizeof(GridBarrier), 0, &ws);
  if (rc == WHTMIX_OK) *err = &static_cast<GridBarrier*>(ws)->err;
  return rc;
}

int done(cudaError_t e) { return e == cudaSuccess ? WHTMIX_OK : host::fail(e); }

bool is_act(int act) { return act >= WHTMIX_ACT_NONE && act <= WHTMIX_ACT_SILU; }

}  // namespace

extern "C" {

int whtmix_rms_norm(const void* x, const void* residual, const float* w, void* h, void* y, float* y_scale, int64_t T, int64_t D,
                    int64_t x_stride, int64_t residual_stride, int64_t h_stride, int64_t y_stride, float eps, int dtype,
                    int out_dtype, void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, D, 1);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_F32 && dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (out_dtype != dtype && out_dtype != WHTMIX_E4M3) return WHTMIX_ERR_BAD_DTYPE;
    if (!(eps >= 0.f)) return WHTMIX_ERR_INVALID_ARG;
    if (T == 0) return WHTMIX_OK;
    const bool q8 = out_dtype == WHTMIX_E4M3;
    if (!x || !w || !y || (q8 && !y_scale)) return WHTMIX_ERR_INVALID_ARG;
    const int es = dtype == WHTMIX_F32 ? 4 : 2;
    if (!residual) h = nullptr;
    const Range out[3] = {{h, T, D, h_stride, es}, {y, T, D, y_stride, q8 ? 1 : es}, {q8 ? y_scale : nullptr, 1, T, T, 4}};
    const Range in[3] = {{x, T, D, x_stride, es}, {residual, T, D, residual_stride, es}, {w, 1, D, D, 4}};
    rc = check_ranges(out, in, [](int o, int i) { return o < 2 && i < 2; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    norm::Forward a{x, residual, w, h, y, y_scale, T, x_stride, residual_stride, h_stride, y_stride, static_cast<int>(D), eps};
    return done(norm::forward(a, dtype == WHTMIX_BF16, q8, sms, static_cast<cudaStream_t>(stream_v)));
  });
}

int whtmix_rms_norm_backward(const void* h, const float* w, const void* dy, const void* dh, void* dx, float* dw, int64_t T, int64_t D,
                             int64_t h_stride, int64_t dy_stride, int64_t dh_stride, int64_t dx_stride, float eps, int dtype,
                             void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, D, 1);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_F32 && dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (!(eps >= 0.f) || !dw) return WHTMIX_ERR_INVALID_ARG;
    if (T > 0 && (!h || !w || !dy || !dx)) return WHTMIX_ERR_INVALID_ARG;
    const int es = dtype == WHTMIX_F32 ? 4 : 2;
    const bool none = T == 0;
    const Range out[2] = {{none ? nullptr : dx, T, D, dx_stride, es}, {dw, 1, D, D, 4}};
    const Range in[4] = {{none ? nullptr : h, T, D, h_stride, es},
                         {none ? nullptr : dy, T, D, dy_stride, es},
                         {none ? nullptr : dh, T, D, dh_stride, es},
                         {none ? nullptr : w, 1, D, D, 4}};
    rc = check_ranges(out, in, [](int o, int i) { return o == 0 && (i == 1 || i == 2); });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (none) return zero(dw, static_cast<size_t>(D) * 4, stream);
    const bool bf16 = dtype == WHTMIX_BF16;
    norm::Backward a{h, w, dy, dh, dx, dw, nullptr, T, h_stride, dy_stride, dh_stride, dx_stride, static_cast<int>(D), eps};
    size_t need = 0;
    rc = done(norm::backward_workspace(a, bf16, sms, &need));
    if (rc == WHTMIX_OK) rc = host::workspace(dev, stream, need, 1, &a.ws);
    if (rc != WHTMIX_OK) return rc;
    return done(norm::backward(a, bf16, sms, stream));
  });
}

int whtmix_linear(const void* x, const void* w, const float* x_scale, const float* w_scale, const float* bias, const void* residual,
                  void* preact, void* y, int64_t T, int64_t N, int64_t K, int64_t x_stride, int64_t w_stride,
                  int64_t residual_stride, int64_t preact_stride, int64_t y_stride, int act, int dtype, int out_dtype,
                  void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, N, K);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_BF16 && dtype != WHTMIX_E4M3) return WHTMIX_ERR_BAD_DTYPE;
    if (out_dtype != WHTMIX_BF16 && out_dtype != WHTMIX_F32) return WHTMIX_ERR_BAD_DTYPE;
    if (!is_act(act)) return WHTMIX_ERR_INVALID_ARG;
    const bool q8 = dtype == WHTMIX_E4M3;
    if (!q8 && (x_scale || w_scale)) return WHTMIX_ERR_INVALID_ARG;
    if (preact && out_dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (T == 0) return WHTMIX_OK;
    if (!x || !w || !y || (q8 && (!x_scale || !w_scale))) return WHTMIX_ERR_INVALID_ARG;
    const int es = q8 ? 1 : 2, os = out_dtype == WHTMIX_F32 ? 4 : 2;
    const Range out[2] = {{y, T, N, y_stride, os}, {preact, T, N, preact_stride, 2}};
    const Range in[6] = {{x, T, K, x_stride, es}, {w, N, K, w_stride, es},   {residual, T, N, residual_stride, os},
                         {bias, 1, N, N, 4},      {x_scale, 1, T, T, 4},     {w_scale, 1, N, N, 4}};
    rc = check_ranges(out, in, [](int o, int i) { return o == 0 && i == 2; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    linear::Forward a{x, w, x_scale, w_scale, bias, residual, preact, y, T, x_stride, w_stride, residual_stride, preact_stride,
                      y_stride, static_cast<int>(K), static_cast<int>(N), act, q8, out_dtype == WHTMIX_F32};
    void* ws = nullptr;
    if (const size_t need = linear::forward_workspace(a, sms)) {
      rc = host::workspace(dev, stream, need, 1, &ws);
      if (rc != WHTMIX_OK) return rc;
    }
    unsigned int* err = nullptr;
    rc = error_word(dev, stream, &err);
    if (rc != WHTMIX_OK) return rc;
    return done(linear::forward(a, ws, err, sms, stream));
  });
}

int whtmix_linear_backward(const void* x, const void* w, const void* dy, const void* preact, void* dx, void* dw, float* db, int64_t T,
                           int64_t N, int64_t K, int64_t x_stride, int64_t w_stride, int64_t dy_stride, int64_t preact_stride,
                           int64_t dx_stride, int act, int dw_dtype, void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, N, K);
    if (rc != WHTMIX_OK) return rc;
    if (dw_dtype != WHTMIX_BF16 && dw_dtype != WHTMIX_F32) return WHTMIX_ERR_BAD_DTYPE;
    if (!is_act(act)) return WHTMIX_ERR_INVALID_ARG;
    const bool none = T == 0;  // (an empty dx may have no address)
    if (!dx && !dw && !db) return none ? WHTMIX_OK : WHTMIX_ERR_INVALID_ARG;
    const int os = dw_dtype == WHTMIX_F32 ? 4 : 2;
    if (!none && (!dy || (dw && !x) || (dx && !w) || (act != WHTMIX_ACT_NONE && !preact))) return WHTMIX_ERR_INVALID_ARG;
    if (act == WHTMIX_ACT_NONE) preact = nullptr;
    const Range out[3] = {{none ? nullptr : dx, T, K, dx_stride, 2}, {dw, N, K, K, os}, {db, 1, N, N, 4}};
    const Range in[4] = {{none || !dw ? nullptr : x, T, K, x_stride, 2},
                         {none || !dx ? nullptr : w, N, K, w_stride, 2},
                         {none ? nullptr : dy, T, N, dy_stride, 2},
                         {none ? nullptr : preact, T, N, preact_stride, 2}};
    rc = check_ranges(out, in, [](int, int) { return false; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (none) {
      rc = zero(dw, static_cast<size_t>(N) * K * os, stream);
      return rc != WHTMIX_OK ? rc : zero(db, static_cast<size_t>(N) * 4, stream);
    }
    linear::Backward a{x, w, dy, preact, dx, dw, db, T, x_stride, w_stride, dy_stride, preact_stride, dx_stride,
                       static_cast<int>(K), static_cast<int>(N), act, dw_dtype == WHTMIX_F32};
    void* ws = nullptr;
    if (const size_t need = linear::backward_workspace(a, sms)) {
      rc = host::workspace(dev, stream, need, 1, &ws);
      if (rc != WHTMIX_OK) return rc;
    }
    unsigned int* err = nullptr;
    rc = error_word(dev, stream, &err);
    if (rc != WHTMIX_OK) return rc;
    return done(linear::backward(a, ws, err, sms, stream));
  });
}

int whtmix_layer_norm(const void* x, const void* residual, const float* w, const float* b, void* h, void* y, float* y_scale, int64_t T,
                      int64_t D, int64_t x_stride, int64_t residual_stride, int64_t h_stride, int64_t y_stride, float eps, int dtype,
                      int out_dtype, void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, D, 1);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_F32 && dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (out_dtype != dtype && out_dtype != WHTMIX_E4M3) return WHTMIX_ERR_BAD_DTYPE;
    if (!(eps >= 0.f)) return WHTMIX_ERR_INVALID_ARG;
    if (T == 0) return WHTMIX_OK;
    const bool q8 = out_dtype == WHTMIX_E4M3;
    if (!x || !w || !y || (q8 && !y_scale)) return WHTMIX_ERR_INVALID_ARG;
    const int es = dtype == WHTMIX_F32 ? 4 : 2;
    if (!residual) h = nullptr;
    const Range out[3] = {{h, T, D, h_stride, es}, {y, T, D, y_stride, q8 ? 1 : es}, {q8 ? y_scale : nullptr, 1, T, T, 4}};
    const Range in[4] = {{x, T, D, x_stride, es}, {residual, T, D, residual_stride, es}, {w, 1, D, D, 4}, {b, 1, D, D, 4}};
    rc = check_ranges(out, in, [](int o, int i) { return o < 2 && i < 2; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    norm::LayerForward a{x, residual, w, b, h, y, y_scale, T, x_stride, residual_stride, h_stride, y_stride, static_cast<int>(D), eps};
    unsigned int* err = nullptr;
    rc = host::error_word(dev, &err);
    if (rc != WHTMIX_OK) return rc;
    return done(norm::layer_forward(a, dtype == WHTMIX_BF16, q8, err, sms, static_cast<cudaStream_t>(stream_v)));
  });
}

int whtmix_layer_norm_backward(const void* h, const float* w, const void* dy, const void* dh, void* dx, float* dw, float* db, int64_t T,
                               int64_t D, int64_t h_stride, int64_t dy_stride, int64_t dh_stride, int64_t dx_stride, float eps, int dtype,
                               void* stream_v) {
  return guarded([&]() -> int {
    int rc = check_sizes(T, D, 1);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_F32 && dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (!(eps >= 0.f) || !dw) return WHTMIX_ERR_INVALID_ARG;
    if (T > 0 && (!h || !w || !dy || !dx)) return WHTMIX_ERR_INVALID_ARG;
    const int es = dtype == WHTMIX_F32 ? 4 : 2;
    const bool none = T == 0;
    const Range out[3] = {{none ? nullptr : dx, T, D, dx_stride, es}, {dw, 1, D, D, 4}, {db, 1, D, D, 4}};
    const Range in[4] = {{none ? nullptr : h, T, D, h_stride, es},
                         {none ? nullptr : dy, T, D, dy_stride, es},
                         {none ? nullptr : dh, T, D, dh_stride, es},
                         {none ? nullptr : w, 1, D, D, 4}};
    rc = check_ranges(out, in, [](int o, int i) { return o == 0 && (i == 1 || i == 2); });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (none) {
      rc = zero(dw, static_cast<size_t>(D) * 4, stream);
      return rc != WHTMIX_OK ? rc : zero(db, static_cast<size_t>(D) * 4, stream);
    }
    const bool bf16 = dtype == WHTMIX_BF16;
    norm::LayerBackward a{h, w, dy, dh, dx, dw, db, nullptr, T, h_stride, dy_stride, dh_stride, dx_stride, static_cast<int>(D), eps};
    size_t need = 0;
    rc = done(norm::layer_backward_workspace(a, bf16, sms, &need));
    if (rc != WHTMIX_OK) return rc;
    host::Scratch scratch;
    rc = scratch.take(dev, stream, need);
    if (rc != WHTMIX_OK) return rc;
    a.ws = scratch.get();
    unsigned int* err = nullptr;
    rc = host::error_word(dev, &err);
    if (rc != WHTMIX_OK) return rc;
    rc = done(norm::layer_backward(a, bf16, err, sms, stream));
    return rc != WHTMIX_OK ? rc : scratch.give_back();
  });
}

int whtmix_gated_linear(const void* x, const void* w, const float* x_scale, const float* w_scale, const float* bias, void* preact, void* y,
                        int64_t T, int64_t N, int64_t K, int64_t x_stride, int64_t w_stride, int64_t preact_stride, int64_t y_stride, int act,
                        int dtype, int out_dtype, void* stream_v) {
  return guarded([&]() -> int {
    if (N < 1) return WHTMIX_ERR_INVALID_ARG;
    if (N > MAX_CHANNELS / 2) return WHTMIX_ERR_BAD_SHAPE;
    int rc = check_sizes(T, 2 * N, K);
    if (rc != WHTMIX_OK) return rc;
    if (dtype != WHTMIX_BF16 && dtype != WHTMIX_E4M3) return WHTMIX_ERR_BAD_DTYPE;
    if (out_dtype != WHTMIX_BF16 && out_dtype != WHTMIX_F32) return WHTMIX_ERR_BAD_DTYPE;
    if (!is_act(act)) return WHTMIX_ERR_INVALID_ARG;
    const bool q8 = dtype == WHTMIX_E4M3;
    if (!q8 && (x_scale || w_scale)) return WHTMIX_ERR_INVALID_ARG;
    if (preact && out_dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
    if (T == 0) return WHTMIX_OK;
    if (!x || !w || !y || (q8 && (!x_scale || !w_scale))) return WHTMIX_ERR_INVALID_ARG;
    const int es = q8 ? 1 : 2, os = out_dtype == WHTMIX_F32 ? 4 : 2;
    const Range out[2] = {{y, T, N, y_stride, os}, {preact, T, 2 * N, preact_stride, 2}};
    const Range in[5] = {{x, T, K, x_stride, es}, {w, 2 * N, K, w_stride, es}, {bias, 1, 2 * N, 2 * N, 4}, {x_scale, 1, T, T, 4}, {w_scale, 1, 2 * N, 2 * N, 4}};
    rc = check_ranges(out, in, [](int, int) { return false; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    linear::Forward a{x, w, x_scale, w_scale, bias, nullptr, preact, y, T, x_stride, w_stride, 0, preact_stride,
                      y_stride, static_cast<int>(K), static_cast<int>(N), act, q8, out_dtype == WHTMIX_F32};
    unsigned int* err = nullptr;
    rc = host::error_word(dev, &err);
    if (rc != WHTMIX_OK) return rc;
    host::Scratch scratch;
    if (const size_t need = linear::gated_forward_workspace(a, sms)) {
      rc = scratch.take(dev, stream, need);
      if (rc != WHTMIX_OK) return rc;
    }
    rc = done(linear::gated_forward(a, scratch.get(), err, sms, stream));
    return rc != WHTMIX_OK ? rc : scratch.give_back();
  });
}

int whtmix_gated_linear_backward(const void* x, const void* w, const void* dy, const void* preact, void* dx, void* dw, float* db, int64_t T,
                                 int64_t N, int64_t K, int64_t x_stride, int64_t w_stride, int64_t dy_stride, int64_t preact_stride,
                                 int64_t dx_stride, int act, int dw_dtype, void* stream_v) {
  return guarded([&]() -> int {
    if (N < 1) return WHTMIX_ERR_INVALID_ARG;
    if (N > MAX_CHANNELS / 2) return WHTMIX_ERR_BAD_SHAPE;
    int rc = check_sizes(T, 2 * N, K);
    if (rc != WHTMIX_OK) return rc;
    if (dw_dtype != WHTMIX_BF16 && dw_dtype != WHTMIX_F32) return WHTMIX_ERR_BAD_DTYPE;
    if (!is_act(act)) return WHTMIX_ERR_INVALID_ARG;
    const bool none = T == 0;  // (an empty dx may have no address)
    if (!dx && !dw && !db) return none ? WHTMIX_OK : WHTMIX_ERR_INVALID_ARG;
    const int os = dw_dtype == WHTMIX_F32 ? 4 : 2;
    if (!none && (!dy || !preact || (dw && !x) || (dx && !w))) return WHTMIX_ERR_INVALID_ARG;
    const Range out[3] = {{none ? nullptr : dx, T, K, dx_stride, 2}, {dw, 2 * N, K, K, os}, {db, 1, 2 * N, 2 * N, 4}};
    const Range in[4] = {{none || !dw ? nullptr : x, T, K, x_stride, 2},
                         {none || !dx ? nullptr : w, 2 * N, K, w_stride, 2},
                         {none ? nullptr : dy, T, N, dy_stride, 2},
                         {none ? nullptr : preact, T, 2 * N, preact_stride, 2}};
    rc = check_ranges(out, in, [](int, int) { return false; });
    if (rc != WHTMIX_OK) return rc;
    int dev = 0, sms = 0;
    rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (none) {
      rc = zero(dw, static_cast<size_t>(2 * N) * K * os, stream);
      return rc != WHTMIX_OK ? rc : zero(db, static_cast<size_t>(2 * N) * 4, stream);
    }
    linear::Backward a{x, w, dy, preact, dx, dw, db, T, x_stride, w_stride, dy_stride, preact_stride, dx_stride,
                       static_cast<int>(K), static_cast<int>(N), act, dw_dtype == WHTMIX_F32};
    unsigned int* err = nullptr;
    rc = host::error_word(dev, &err);
    if (rc != WHTMIX_OK) return rc;
    host::Scratch scratch;
    if (const size_t need = linear::gated_backward_workspace(a, sms)) {
      rc = scratch.take(dev, stream, need);
      if (rc != WHTMIX_OK) return rc;
    }
    rc = done(linear::gated_backward(a, scratch.get(), err, sms, stream));
    return rc != WHTMIX_OK ? rc : scratch.give_back();
  });
}

static int global_norm(const whtmix_tensor_t* tensors, int64_t count, float max_norm, float* norm, bool scale, void* stream_v) {
  return guarded([&]() -> int {
    if (count < 0 || (count > 0 && !tensors) || (!norm && !scale)) return WHTMIX_ERR_INVALID_ARG;
    if (scale && !(max_norm >= 0.f)) return WHTMIX_ERR_INVALID_ARG;
    if (count > MAX_TENSORS) return WHTMIX_ERR_BAD_SHAPE;
    if (reinterpret_cast<uintptr_t>(norm) & 3u) return WHTMIX_ERR_MISALIGNED;
    // what is read and written, by address: an output may overlap nothing but its own input, whole
    struct Span {
      uintptr_t lo, hi;
      bool out;
    };
    std::vector<clip::Item> items;
    std::vector<Span> spans;
    items.reserve(static_cast<size_t>(count));
    spans.reserve(2 * static_cast<size_t>(count) + 1);
    auto span = [&](const void* p, size_t bytes, bool out) {
      const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
      spans.push_back({lo, lo + bytes, out});
    };
    for (int64_t i = 0; i < count; ++i) {
      const whtmix_tensor_t& t = tensors[i];
      if (t.dtype != WHTMIX_F32 && t.dtype != WHTMIX_BF16) return WHTMIX_ERR_BAD_DTYPE;
      if (t.n < 0) return WHTMIX_ERR_INVALID_ARG;
      if (t.n > MAX_ELEMENTS) return WHTMIX_ERR_BAD_SHAPE;
      if (t.n == 0) continue;
      if (!t.in || (scale && !t.out)) return WHTMIX_ERR_INVALID_ARG;
      const size_t es = t.dtype == WHTMIX_F32 ? 4 : 2;
      if ((reinterpret_cast<uintptr_t>(t.in) | (scale ? reinterpret_cast<uintptr_t>(t.out) : 0)) & (es - 1)) return WHTMIX_ERR_MISALIGNED;
      items.push_back({t.in, scale ? t.out : nullptr, t.n, t.dtype == WHTMIX_BF16});
      if (!scale || t.in != t.out) span(t.in, t.n * es, false);
      if (scale) span(t.out, t.n * es, true);
    }
    if (norm) span(norm, 4, true);
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    uintptr_t end = 0, end_out = 0;  // of those before: all, and the outputs
    for (const Span& s : spans) {
      if (s.lo < (s.out ? end : end_out)) return WHTMIX_ERR_ALIAS;
      end = std::max(end, s.hi);
      if (s.out) end_out = std::max(end_out, s.hi);
    }
    if (items.empty() && !norm) return WHTMIX_OK;
    int dev = 0, sms = 0;
    int rc = host::device(&dev, &sms);
    if (rc != WHTMIX_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (items.empty()) return zero(norm, 4, stream);
    const clip::Call a{items.data(), static_cast<long long>(items.size()), norm, max_norm, scale};
    host::Scratch scratch;
    if (const size_t need = clip::workspace(a, sms)) {
      rc = scratch.take(dev, stream, need);
      if (rc != WHTMIX_OK) return rc;
    }
    rc = done(clip::run(a, scratch.get(), sms, stream));
    return rc != WHTMIX_OK ? rc : scratch.give_back();
  });
}

int whtmix_global_norm(const whtmix_tensor_t* tensors, int64_t count, float* norm, void* stream_v) {
  return global_norm(tensors, count, 0.f, norm, false, stream_v);
}

int whtmix_clip_by_global_norm(const whtmix_tensor_t* tensors, int64_t count, float max_norm, float* norm, void* stream_v) {
  return global_norm(tensors, count, max_norm, norm, true, stream_v);
}

}  // extern "C"
