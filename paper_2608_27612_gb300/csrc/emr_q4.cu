// Matrices in 4 bits with a scale for each group of a row's columns: laid out from a matrix or from given codes,
// and given back. A warp takes a row's 128 columns, four a lane; two lanes' codes make a word. Done once for a
// layer, and kept simple: elements are loaded one by one, and places are found by division, so that it is bound by instructions and
// the latency of its loads. 8192 x 8192 in groups of 32: from bfloat16 210 us (0.8 TB/s), from its transpose, whose elements lie in
// lines of their own, 248, from codes 179, back to bfloat16 123.
#include "emr_q4.h"

namespace {

using namespace emr;

struct Args {
  const void* src;
  const __nv_bfloat16* scales;
  int32_t dtype, group;
  int64_t rows, cols, batch_stride, row_stride, col_stride, s_batch, s_row, s_col;
  int64_t tiles, blocks, total;  // total: rows of units (16 rows each), blocks, of all matrices, in rows x blocks
  uint8_t* data;
  void* out;
};

__device__ __forceinline__ float load_value(const void* p, int dtype, int64_t i) {
  if (dtype == EMR_F32) return static_cast<const float*>(p)[i];
  if (dtype == EMR_BF16) return float(static_cast<const __nv_bfloat16*>(p)[i]);
  return float(static_cast<const __half*>(p)[i]);
}

// kFrom: 0 a matrix, quantised; 1 codes and scales; 2 back to a matrix.
template <int kFrom>
__global__ void __launch_bounds__(256) q4_kernel(const __grid_constant__ Args a) {
  const int lane = threadIdx.x & 31;
  const int per = kQ4Cols / a.group;
  for (int64_t at = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); at < a.total; at += int64_t(gridDim.x) * 8) {
    // blocks fastest, then rows, then matrices
    const int64_t kb = at % a.blocks, line = at / a.blocks, row = line % (a.tiles * kQ4Rows), b = line / (a.tiles * kQ4Rows);
    uint8_t* const unit = a.data + ((b * a.tiles + row / kQ4Rows) * a.blocks + kb) * q4_unit(a.group);
    const int r = int(row % kQ4Rows), in_block = lane * 4 / a.group;
    uint32_t* const word = reinterpret_cast<uint32_t*>(unit + q4_word_at(r, lane));
    __nv_bfloat16* const scale_at = reinterpret_cast<__nv_bfloat16*>(unit + q4_scale_at(r, in_block, a.group));
    const int64_t col = kb * kQ4Cols + lane * 4;
    if (kFrom == 2) {
      if (row >= a.rows) continue;
      const uint32_t w = *word >> q4_shift(lane);
      const float scale = float(*scale_at);
      const int shifts[4] = {0, 16, 4, 20};
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (col + j < a.cols) store_scalar(a.out, a.dtype, (b * a.rows + row) * a.cols + col + j, scale * float(int(w >> shifts[j] & 15) - 8));
      continue;
    }
    int c[4];
    float scale = 0.f;
    if (kFrom == 0) {
      float v[4], top = 0.f;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        v[j] = row < a.rows && col + j < a.cols ? load_value(a.src, a.dtype, b * a.batch_stride + row * a.row_stride + (col + j) * a.col_stride) : 0.f;
        top = fmaxf(top, isfinite(v[j]) ? fabsf(v[j]) : INFINITY);
      }
      for (int o = a.group / 8; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      scale = float(__float2bfloat16_rn(__fdiv_rn(top, 7.f)));
      if (scale < 0x1p-126f) scale = 0.f;  // the whole group is held as 0
      if (!(scale < INFINITY)) scale = NAN;
#pragma unroll
      for (int j = 0; j < 4; j++) c[j] = scale > 0.f ? max(-8, min(7, __float2int_rn(__fdiv_rn(v[j], scale)))) : 0;
    } else {
      const int8_t* const codes = static_cast<const int8_t*>(a.src);
#pragma unroll
      for (int j = 0; j < 4; j++)
        c[j] = row < a.rows && col + j < a.cols ? codes[b * a.batch_stride + row * a.row_stride + (col + j) * a.col_stride] : 0;
      const int64_t g = kb * per + in_block;
      if (row < a.rows && g * a.group < a.cols) scale = float(a.scales[b * a.s_batch + row * a.s_row + g * a.s_col]);
    }
    uint32_t w = q4_place(c[0], c[1], c[2], c[3], q4_shift(lane));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    if (!(lane & 1)) *word = w;
    if (lane * 4 % a.group == 0) *scale_at = __float2bfloat16_rn(scale);
  }
}

template <int kFrom>
emr_status launch(Args a, const emr_q4* q, cudaStream_t st) {
  a.group = q->group, a.rows = q->rows, a.cols = q->cols, a.data = q->data;
  a.tiles = q4_tiles(q->rows), a.blocks = q4_blocks(q->cols);
  a.total = int64_t(q->batch) * a.tiles * kQ4Rows * a.blocks;
  const int64_t blocks = (a.total + 7) / 8;
  return launch_plain(q4_kernel<kFrom>, dim3(unsigned(blocks < (1 << 20) ? blocks : 1 << 20)), 256, st, a);
}

emr_status sizes_ok(const emr_q4* q, size_t* bytes) {
  if (!q4_ok(q)) return EMR_ERR_ARG;
  return emr_q4_size(q->batch, q->rows, q->cols, q->group, bytes);
}
// Whether matrices of q's rows and `cols` columns with these strides lie in q's memory.
bool in_data(const emr_q4* q, size_t bytes, const void* p, int size, int64_t cols, int64_t batch_stride, int64_t row_stride, int64_t col_stride) {
  return overlap(q->data, int64_t(bytes), 1, p, (q->batch - 1) * batch_stride + (q->rows - 1) * row_stride + (cols - 1) * col_stride + 1, size);
}

}  // namespace

extern "C" emr_status emr_q4_size(int32_t batch, int64_t rows, int64_t cols, int32_t group, size_t* bytes) {
  if (batch < 1 || rows < 1 || cols < 1 || !bytes || (group != 32 && group != 64 && group != 128)) return EMR_ERR_ARG;
  if (rows > kQ8MaxDim || cols > kQ8MaxDim) return EMR_ERR_RANGE;
  const double size = double(batch) * double(q4_tiles(rows)) * double(q4_blocks(cols)) * q4_unit(group);
  if (size > 1e18) return EMR_ERR_RANGE;
  *bytes = size_t(batch) * size_t(q4_tiles(rows)) * size_t(q4_blocks(cols)) * size_t(q4_unit(group));
  return EMR_OK;
}

extern "C" emr_status emr_q4_quantize(const void* src, int32_t dtype, int64_t batch_stride, int64_t row_stride, int64_t col_stride,
                                      const emr_q4* q, void* stream) {
  size_t bytes;
  const emr_status ok = sizes_ok(q, &bytes);
  if (ok != EMR_OK) return ok;
  if (!src || !dtype_ok(dtype) || reinterpret_cast<uintptr_t>(src) % dtype_bytes(dtype) || batch_stride < 0 || row_stride < 0 || col_stride < 0 ||
      in_data(q, bytes, src, dtype_bytes(dtype), q->cols, batch_stride, row_stride, col_stride))
    return EMR_ERR_ARG;
  Args a{};
  a.src = src, a.dtype = dtype, a.batch_stride = batch_stride, a.row_stride = row_stride, a.col_stride = col_stride;
  return launch<0>(a, q, static_cast<cudaStream_t>(stream));
}

extern "C" emr_status emr_q4_pack(const int8_t* codes, int64_t batch_stride, int64_t row_stride, int64_t col_stride, const void* scales,
                                  int64_t s_batch, int64_t s_row, int64_t s_col, const emr_q4* q, void* stream) {
  size_t bytes;
  const emr_status ok = sizes_ok(q, &bytes);
  if (ok != EMR_OK) return ok;
  if (!codes || !scales || reinterpret_cast<uintptr_t>(scales) % 2 || batch_stride < 0 || row_stride < 0 || col_stride < 0 || s_batch < 0 ||
      s_row < 0 || s_col < 0 || in_data(q, bytes, codes, 1, q->cols, batch_stride, row_stride, col_stride) ||
      in_data(q, bytes, scales, 2, (q->cols + q->group - 1) / q->group, s_batch, s_row, s_col))
    return EMR_ERR_ARG;
  Args a{};
  a.src = codes, a.batch_stride = batch_stride, a.row_stride = row_stride, a.col_stride = col_stride;
  a.scales = static_cast<const __nv_bfloat16*>(scales), a.s_batch = s_batch, a.s_row = s_row, a.s_col = s_col;
  return launch<1>(a, q, static_cast<cudaStream_t>(stream));
}

extern "C" emr_status emr_q4_dequantize(const emr_q4* q, void* out, int32_t dtype, void* stream) {
  size_t bytes;
  const emr_status ok = sizes_ok(q, &bytes);
  if (ok != EMR_OK) return ok;
  if (!out || !dtype_ok(dtype) || reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype) ||
      in_data(q, bytes, out, dtype_bytes(dtype), q->cols, q->rows * q->cols, q->cols, 1))
    return EMR_ERR_ARG;
  Args a{};
  a.dtype = dtype, a.out = out;
  return launch<2>(a, q, static_cast<cudaStream_t>(stream));
}
