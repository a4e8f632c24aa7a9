// Dense layers in 8 bits: each pass of a layer as one call on the caller's memory, made of the
// quantising kernels and the matrix product. Host code only.
#include <cuda_runtime.h>

#include "emr_q8.h"

namespace {

using namespace emr;

size_t value_bytes(int64_t batch, int64_t rows, int64_t cols) { return size_t(batch) * rows * q8_row_bytes(cols); }
size_t packed_bytes(int64_t batch, int64_t rows, int64_t cols) {
  return value_bytes(batch, rows, cols) + size_t(batch) * q8_scale_batch(rows, cols);
}
// An 8-bit matrix in one piece of memory: values, then scales.
emr_q8 packed(void* p, int64_t batch, int64_t rows, int64_t cols) {
  uint8_t* v = static_cast<uint8_t*>(p);
  return {int32_t(batch), 0, rows, cols, v, v + value_bytes(batch, rows, cols)};
}
bool layer_ok(const emr_dense* l) { return l && q8_ok(&l->w) && l->act >= EMR_ACT_IDENTITY && l->act <= EMR_ACT_ABS; }
// Sizes for which the byte counts below fit their types.
emr_status check(const emr_dense* l, int32_t x_batch, int64_t rows) {
  if (!layer_ok(l) || rows < 1 || (x_batch != 1 && x_batch != l->w.batch)) return EMR_ERR_ARG;
  size_t v, s;
  const emr_status a = emr_q8_size(l->w.batch, rows, l->w.cols, &v, &s);
  if (a != EMR_OK) return a;
  return emr_q8_size(l->w.batch, rows, l->w.rows, &v, &s);
}
size_t padded(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

extern "C" emr_status emr_dense_forward_room(const emr_dense* layer, int32_t x_batch, int64_t rows, int32_t keep, size_t* x_bytes,
                                             size_t* xt_bytes, size_t* slope_bytes) {
  if (!x_bytes || !xt_bytes || !slope_bytes) return EMR_ERR_ARG;
  const emr_status s = check(layer, x_batch, rows);
  if (s != EMR_OK) return s;
  *x_bytes = !keep && few_fused(rows, layer->w) ? 0 : packed_bytes(x_batch, rows, layer->w.cols);
  *xt_bytes = keep ? packed_bytes(x_batch, layer->w.cols, rows) : 0;
  *slope_bytes = keep && layer->act != EMR_ACT_IDENTITY ? packed_bytes(layer->w.batch, rows, layer->w.rows) : 0;
  return EMR_OK;
}

extern "C" emr_status emr_dense_forward(const emr_dense* layer, const void* x, int32_t dtype, int32_t x_batch, int64_t rows,
                                        int64_t batch_stride, int64_t row_stride, int64_t col_stride, void* out, int32_t out_dtype,
                                        int32_t keep, void* x8, void* xt, void* slope, void* stream) {
  size_t x_bytes = 0, xt_bytes = 0, slope_bytes = 0;
  const emr_status s = emr_dense_forward_room(layer, x_batch, rows, keep, &x_bytes, &xt_bytes, &slope_bytes);
  if (s != EMR_OK) return s;
  if (!x || !out || !dtype_ok(dtype) || !dtype_ok(out_dtype) || batch_stride < 0 || row_stride < 0 || col_stride < 0 ||
      (x_bytes && !x8) || (xt_bytes && !xt) || (slope_bytes && !slope))
    return EMR_ERR_ARG;
  if (!x_bytes) {
    const int size = dtype_bytes(dtype), out_size = dtype_bytes(out_dtype);
    if (reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(out) % out_size ||
        reinterpret_cast<uintptr_t>(layer->bias) % 4)
      return EMR_ERR_ARG;
    FewArgs f{};
    f.x = x, f.x_dtype = dtype, f.x_batch = x_batch, f.x_rows = rows;
    f.x_batch_stride = batch_stride, f.x_row_stride = row_stride, f.x_col_stride = col_stride;
    f.w = &layer->w, f.bias = layer->bias, f.act = layer->act, f.out = out, f.out_dtype = out_dtype, f.batch = layer->w.batch;
    return launch_few(f, static_cast<cudaStream_t>(stream));
  }
  const emr_q8 q = packed(x8, x_batch, rows, layer->w.cols);
  const emr_q8 t = packed(xt, x_batch, layer->w.cols, rows);
  const emr_status e =
      keep ? emr_q8_quantize_held(x, dtype, x_batch, rows, layer->w.cols, batch_stride, row_stride, col_stride, &q, &t, stream)
           : emr_q8_quantize(x, dtype, x_batch, rows, layer->w.cols, batch_stride, row_stride, col_stride, &q, nullptr, stream);
  if (e != EMR_OK) return e;
  const emr_q8 d = packed(slope, layer->w.batch, rows, layer->w.rows);
  return emr_q8_matmul(&q, &layer->w, layer->bias, layer->act, 0, out, out_dtype, slope_bytes ? &d : nullptr, stream);
}

extern "C" emr_status emr_dense_backward_room(const emr_dense* layer, int32_t x_batch, int64_t rows, size_t* bytes) {
  if (!bytes) return EMR_ERR_ARG;
  const emr_status s = check(layer, x_batch, rows);
  if (s != EMR_OK) return s;
  const int64_t nets = layer->w.batch, n = layer->w.rows;
  size_t sums = 0;
  const emr_status e = emr_q8_slope_workspace_size(int32_t(nets), rows, n, &sums);
  if (e != EMR_OK) return e;
  *bytes = padded(packed_bytes(nets, rows, n)) + padded(packed_bytes(nets, n, rows)) + sums;
  return EMR_OK;
}

extern "C" emr_status emr_dense_backward(const emr_dense* layer, const void* dy, int32_t dtype, int32_t x_batch, int64_t rows,
                                         const void* xt, const void* slope, void* dx, void* dw, void* db, int32_t out_dtype,
                                         void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  emr_status s = emr_dense_backward_room(layer, x_batch, rows, &need);
  if (s != EMR_OK) return s;
  if (!dy || (dw && !xt) || !ws || !dtype_ok(dtype) || !dtype_ok(out_dtype) || (!dx && !dw && !db) ||
      (layer->act != EMR_ACT_IDENTITY && !slope) || (dx && !q8_ok(&layer->wt)) || reinterpret_cast<uintptr_t>(ws) % 16)
    return EMR_ERR_ARG;
  const int64_t nets = layer->w.batch, n = layer->w.rows, k = layer->w.cols;
  if (dx && (layer->wt.batch != nets || layer->wt.rows != k || layer->wt.cols != n)) return EMR_ERR_ARG;
  if (ws_bytes < need) return EMR_ERR_CAPACITY;
  uint8_t* p = static_cast<uint8_t*>(ws);
  const emr_q8 dz = packed(p, nets, rows, n);
  p += padded(packed_bytes(nets, rows, n));
  const emr_q8 dzt = packed(p, nets, n, rows);
  p += padded(packed_bytes(nets, n, rows));
  const emr_q8 x = packed(const_cast<void*>(xt), x_batch, k, rows), d = packed(const_cast<void*>(slope), nets, rows, n);
  s = emr_q8_slope(dy, dtype, int32_t(nets), rows, n, layer->act != EMR_ACT_IDENTITY ? &d : nullptr, dx ? &dz : nullptr,
                   dw ? &dzt : nullptr, db, out_dtype, p, ws_bytes - size_t(p - static_cast<uint8_t*>(ws)), stream);
  if (s != EMR_OK) return s;
  if (dx) {
    s = emr_q8_matmul(&dz, &layer->wt, nullptr, EMR_ACT_IDENTITY, x_batch < nets, dx, out_dtype, nullptr, stream);
    if (s != EMR_OK) return s;
  }
  if (dw) s = emr_q8_matmul(&dzt, &x, nullptr, EMR_ACT_IDENTITY, 0, dw, out_dtype, nullptr, stream);
  return s;
}
