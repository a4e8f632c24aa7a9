// Block-scaled 8-bit matrices: quantising, transposing, reading back, and the
// backward pass of an activation from its 8-bit slope.
//
// All of it is bound by memory. Every kernel reads its source once: a row block of
// 128 columns is one warp's registers (four columns a lane), so its maximum is one
// warp reduction and its codes one 128-byte store. The transposed copy goes through
// a 64 KB tile in shared memory whose 16-byte columns are exchanged by (row / 4) % 8,
// which makes both the row-wise stores and the column-wise loads (a lane takes four
// rows x four columns) free of bank conflicts.
#include <cuda_runtime.h>

#include "emr_q8.h"

namespace {

using namespace emr;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint32_t magnitude4(float4 v) {
  return max(max(q8_magnitude(v.x), q8_magnitude(v.y)), max(q8_magnitude(v.z), q8_magnitude(v.w)));
}

// Sources: four columns c .. c + 3 of row r, zero past the matrix.
struct DenseSource {
  const void* p;
  int dtype;
  int64_t row_stride, col_stride;
  bool vector;  // col_stride 1 and every row aligned to four elements
  __device__ __forceinline__ float4 four(int64_t base, int64_t r, int64_t c, int64_t cols) const {
    const int64_t at = base + r * row_stride;
    if (vector && c + 4 <= cols) return load_four(p, dtype, at + c);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < cols) v.x = load_scalar(p, dtype, at + c * col_stride);
    if (c + 1 < cols) v.y = load_scalar(p, dtype, at + (c + 1) * col_stride);
    if (c + 2 < cols) v.z = load_scalar(p, dtype, at + (c + 2) * col_stride);
    if (c + 3 < cols) v.w = load_scalar(p, dtype, at + (c + 3) * col_stride);
    return v;
  }
};

__device__ __forceinline__ float4 q8_four(const uint8_t* values, const uint8_t* scales, int64_t row_bytes,
                                          int64_t chunks, int64_t r, int64_t c) {
  const float s = q8_scale(scales[q8_scale_at(chunks, r, c >> 7)]);
  const float4 v = q8_unpack4(*reinterpret_cast<const uint32_t*>(values + r * row_bytes + c));
  return make_float4(v.x * s, v.y * s, v.z * s, v.w * s);
}

// Row blocks only: one warp takes four blocks of 128 columns of one row, whose four
// scale bytes are one word.
__global__ void __launch_bounds__(kThreads) q8_rows_kernel(DenseSource src, int64_t batch_stride, int64_t rows,
                                                           int64_t cols, int64_t units, emr_q8 q) {
  const int64_t chunks = q8_scale_chunks(cols), blocks = q8_blocks(cols), row_bytes = q8_row_bytes(cols);
  const int64_t unit = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (unit >= units) return;
  const int lane = threadIdx.x & 31;
  const int64_t chunk = unit % chunks, row = unit / chunks, b = row / rows, r = row - b * rows;
  float4 v[4];
#pragma unroll
  for (int j = 0; j < 4; j++) v[j] = src.four(b * batch_stride, r, (chunk * 4 + j) * 128 + lane * 4, cols);
  uint8_t* out = q.values + (b * rows + r) * row_bytes;
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const uint32_t byte = q8_scale_byte(warp_max(magnitude4(v[j])));
    word |= byte << (8 * j);
    if (chunk * 4 + j < blocks)
      *reinterpret_cast<uint32_t*>(out + (chunk * 4 + j) * 128 + lane * 4) =
          q8_pack4(v[j].x, v[j].y, v[j].z, v[j].w, q8_inverse(byte));
  }
  if (lane == 0)
    *reinterpret_cast<uint32_t*>(q.scales + b * q8_scale_batch(rows, cols) + q8_scale_at(chunks, r, chunk * 4)) = word;
}

// One 128 x 128 tile: row blocks to q, column blocks (the transpose) to qt, column
// sums to sums[b][row tile][cols]. Mode 0: a dense source; 1: the values of an 8-bit
// matrix; 2: the product of a dense matrix and an 8-bit one.
template <int kMode>
__global__ void __launch_bounds__(kThreads) q8_tile_kernel(DenseSource src, int64_t batch_stride, emr_q8 other,
                                                           int64_t rows, int64_t cols, emr_q8 q, emr_q8 qt,
                                                           float* sums) {
  extern __shared__ float4 tile[];  // [128][32]
  const int64_t row_tiles = q8_blocks(rows), col_tiles = q8_blocks(cols);
  const int64_t ct = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles, rt = rest % row_tiles, b = rest / row_tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t chunks = q8_scale_chunks(cols), row_bytes = q8_row_bytes(cols), scale_batch = q8_scale_batch(rows, cols);
  const int64_t c = ct * 128 + lane * 4;
  uint8_t* qv = q.values ? q.values + b * rows * row_bytes : nullptr;
  uint8_t* qs = q.values ? q.scales + b * scale_batch : nullptr;
#pragma unroll 4
  for (int i = warp; i < 128; i += kWarps) {
    const int64_t r = rt * 128 + i;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows) {
      if (kMode != 1) v = src.four(b * batch_stride, r, c, cols);
      if (kMode != 0) {
        const float4 u = q8_four(other.values + b * rows * row_bytes, other.scales + b * scale_batch, row_bytes, chunks, r, c);
        // one rounding each, so that the values are those of the plain product
        v = kMode == 1 ? u : make_float4(__fmul_rn(v.x, u.x), __fmul_rn(v.y, u.y), __fmul_rn(v.z, u.z), __fmul_rn(v.w, u.w));
      }
    }
    if (qv && r < rows) {
      const uint32_t byte = q8_scale_byte(warp_max(magnitude4(v)));
      *reinterpret_cast<uint32_t*>(qv + r * row_bytes + c) = q8_pack4(v.x, v.y, v.z, v.w, q8_inverse(byte));
      if (lane == 0) qs[q8_scale_at(chunks, r, ct)] = uint8_t(byte);
    }
    if (qt.values || sums) tile[i * 32 + (lane ^ ((i >> 2) & 7))] = v;
  }
  if (!qt.values && !sums) return;
  __syncthreads();
  const int64_t t_chunks = q8_scale_chunks(rows), t_row_bytes = q8_row_bytes(rows);
  uint8_t* tv = qt.values ? qt.values + b * cols * t_row_bytes : nullptr;
  uint8_t* ts = qt.values ? qt.scales + b * q8_scale_batch(cols, rows) : nullptr;
  for (int i = warp; i < 32; i += kWarps) {  // columns 4 i .. 4 i + 3, rows 4 lane .. 4 lane + 3
    float4 v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = tile[(lane * 4 + j) * 32 + (i ^ (lane & 7))];
    const float col[4][4] = {{v[0].x, v[1].x, v[2].x, v[3].x}, {v[0].y, v[1].y, v[2].y, v[3].y},
                             {v[0].z, v[1].z, v[2].z, v[3].z}, {v[0].w, v[1].w, v[2].w, v[3].w}};
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const int64_t n = ct * 128 + i * 4 + j;
      if (tv) {
        const uint32_t byte = q8_scale_byte(warp_max(magnitude4(make_float4(col[j][0], col[j][1], col[j][2], col[j][3]))));
        if (n < cols) {
          *reinterpret_cast<uint32_t*>(tv + n * t_row_bytes + rt * 128 + lane * 4) =
              q8_pack4(col[j][0], col[j][1], col[j][2], col[j][3], q8_inverse(byte));
          if (lane == 0) ts[q8_scale_at(t_chunks, n, rt)] = uint8_t(byte);
        }
      }
      if (sums) {
        float s = (col[j][0] + col[j][1]) + (col[j][2] + col[j][3]);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0 && n < cols) sums[(b * row_tiles + rt) * cols + n] = s;
      }
    }
  }
}

// Sum of the row tiles' column sums, in the order of the tiles.
__global__ void __launch_bounds__(kThreads) q8_sums_kernel(const float* sums, int64_t row_tiles, int64_t cols,
                                                           int64_t total, void* db, int dtype) {
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= total) return;
  const int64_t b = i / cols, n = i - b * cols;
  const float* p = sums + b * row_tiles * cols + n;
  float s = 0.f;
  for (int64_t t = 0; t < row_tiles; t++) s += p[t * cols];
  store_scalar(db, dtype, i, s);
}

__global__ void __launch_bounds__(kThreads) q8_dequantize_kernel(emr_q8 q, int64_t total, void* out, int dtype) {
  const int64_t row_bytes = q8_row_bytes(q.cols), quads = row_bytes / 4;
  const int64_t chunks = q8_scale_chunks(q.cols), scale_batch = q8_scale_batch(q.rows, q.cols);
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kThreads) {
    const int64_t row = i / quads, c = (i - row * quads) * 4, b = row / q.rows, r = row - b * q.rows;
    const float4 v = q8_four(q.values + b * q.rows * row_bytes, q.scales + b * scale_batch, row_bytes, chunks, r, c);
    const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (c + j < q.cols) store_scalar(out, dtype, row * q.cols + c + j, e[j]);
  }
}

constexpr int64_t kMaxGrid = (int64_t(1) << 31) - 1;
constexpr int kTileBytes = 128 * 128 * 4;

template <int kMode>
emr_status launch_tile(const DenseSource& src, int64_t batch_stride, const emr_q8* other, int64_t batch, int64_t rows,
                       int64_t cols, const emr_q8* q, const emr_q8* qt, float* sums, cudaStream_t st) {
  const int64_t tiles = batch * q8_blocks(rows) * q8_blocks(cols);
  if (tiles > kMaxGrid) return EMR_ERR_RANGE;
  const int smem = qt || sums ? kTileBytes : 0;
  if (smem && cudaFuncSetAttribute(q8_tile_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return EMR_ERR_CUDA;
  const emr_q8 none{};
  q8_tile_kernel<kMode><<<unsigned(tiles), kThreads, smem, st>>>(src, batch_stride, other ? *other : none, rows, cols,
                                                                 q ? *q : none, qt ? *qt : none, sums);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

bool same_shape(const emr_q8* q, int64_t batch, int64_t rows, int64_t cols) {
  return q8_ok(q) && q->batch == batch && q->rows == rows && q->cols == cols;
}

}  // namespace

extern "C" emr_status emr_q8_size(int32_t batch, int64_t rows, int64_t cols, size_t* value_bytes, size_t* scale_bytes) {
  if (!value_bytes || !scale_bytes || batch < 1 || rows < 1 || cols < 1) return EMR_ERR_ARG;
  if (rows > kQ8MaxDim || cols > kQ8MaxDim) return EMR_ERR_RANGE;
  const __int128 v = __int128(batch) * rows * q8_row_bytes(cols), s = __int128(batch) * q8_scale_batch(rows, cols);
  if (v > INT64_MAX || s > INT64_MAX) return EMR_ERR_RANGE;
  *value_bytes = size_t(v);
  *scale_bytes = size_t(s);
  return EMR_OK;
}

extern "C" emr_status emr_q8_quantize(const void* src, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                                      int64_t batch_stride, int64_t row_stride, int64_t col_stride, const emr_q8* q,
                                      const emr_q8* qt, void* stream) {
  if (!src || !dtype_ok(dtype) || batch < 1 || rows < 1 || cols < 1 || batch_stride < 0 || row_stride < 0 ||
      col_stride < 0 || (!q && !qt))
    return EMR_ERR_ARG;
  if (rows > kQ8MaxDim || cols > kQ8MaxDim) return EMR_ERR_RANGE;
  if ((q && !same_shape(q, batch, rows, cols)) || (qt && !same_shape(qt, batch, cols, rows))) return EMR_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(src) % dtype_bytes(dtype)) return EMR_ERR_ARG;
  if (row_stride == 1 && col_stride != 1) {  // column-major: the same matrix seen as its transpose
    const int64_t r = rows, s = row_stride;
    rows = cols, cols = r, row_stride = col_stride, col_stride = s;
    const emr_q8* t = q;
    q = qt, qt = t;
  }
  const int size = dtype_bytes(dtype);
  DenseSource d{src, dtype, row_stride, col_stride, false};
  d.vector = col_stride == 1 && reinterpret_cast<uintptr_t>(src) % (4 * size) == 0 && (rows == 1 || row_stride % 4 == 0) &&
             (batch == 1 || batch_stride % 4 == 0);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (qt) return launch_tile<0>(d, batch_stride, nullptr, batch, rows, cols, q, qt, nullptr, st);
  const int64_t units = int64_t(batch) * rows * q8_scale_chunks(cols), grid = (units + kWarps - 1) / kWarps;
  if (grid > kMaxGrid) return EMR_ERR_RANGE;
  q8_rows_kernel<<<unsigned(grid), kThreads, 0, st>>>(d, batch_stride, rows, cols, units, *q);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

extern "C" emr_status emr_q8_transpose(const emr_q8* q, const emr_q8* qt, void* stream) {
  if (!q8_ok(q) || !same_shape(qt, q->batch, q->cols, q->rows)) return EMR_ERR_ARG;
  return launch_tile<1>(DenseSource{}, 0, q, q->batch, q->rows, q->cols, nullptr, qt, nullptr,
                        static_cast<cudaStream_t>(stream));
}

extern "C" emr_status emr_q8_dequantize(const emr_q8* q, void* out, int32_t dtype, void* stream) {
  if (!q8_ok(q) || !out || !dtype_ok(dtype) || reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype)) return EMR_ERR_ARG;
  const int64_t total = q->batch * q->rows * (q8_row_bytes(q->cols) / 4);
  const int64_t grid = (total + kThreads - 1) / kThreads;
  q8_dequantize_kernel<<<unsigned(grid < (1 << 20) ? grid : (1 << 20)), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      *q, total, out, dtype);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

extern "C" emr_status emr_q8_slope_workspace_size(int32_t batch, int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes || batch < 1 || rows < 1 || cols < 1) return EMR_ERR_ARG;
  if (rows > kQ8MaxDim || cols > kQ8MaxDim) return EMR_ERR_RANGE;
  const __int128 n = __int128(batch) * q8_blocks(rows) * cols * 4;
  if (n > INT64_MAX) return EMR_ERR_RANGE;
  *bytes = size_t(n);
  return EMR_OK;
}

extern "C" emr_status emr_q8_slope(const void* dy, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                                   const emr_q8* d, const emr_q8* dz, const emr_q8* dzt, void* db, int32_t db_dtype,
                                   void* ws, size_t ws_bytes, void* stream) {
  if (!dy || !dtype_ok(dtype) || (!dz && !dzt && !db) || (db && (!dtype_ok(db_dtype) || !ws))) return EMR_ERR_ARG;
  size_t need = 0;
  const emr_status s = emr_q8_slope_workspace_size(batch, rows, cols, &need);
  if (s != EMR_OK) return s;
  if ((d && !same_shape(d, batch, rows, cols)) || (dz && !same_shape(dz, batch, rows, cols)) ||
      (dzt && !same_shape(dzt, batch, cols, rows)))
    return EMR_ERR_ARG;
  const int size = dtype_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(dy) % size || (db && (reinterpret_cast<uintptr_t>(db) % dtype_bytes(db_dtype) ||
                                                        reinterpret_cast<uintptr_t>(ws) % 4)))
    return EMR_ERR_ARG;
  if (db && ws_bytes < need) return EMR_ERR_CAPACITY;
  DenseSource src{dy, dtype, cols, 1, false};
  src.vector = reinterpret_cast<uintptr_t>(dy) % (4 * size) == 0 && cols % 4 == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  float* sums = db ? static_cast<float*>(ws) : nullptr;
  const emr_status e = d ? launch_tile<2>(src, rows * cols, d, batch, rows, cols, dz, dzt, sums, st)
                         : launch_tile<0>(src, rows * cols, nullptr, batch, rows, cols, dz, dzt, sums, st);
  if (e != EMR_OK || !db) return e;
  const int64_t total = int64_t(batch) * cols, grid = (total + kThreads - 1) / kThreads;
  if (grid > kMaxGrid) return EMR_ERR_RANGE;
  q8_sums_kernel<<<unsigned(grid), kThreads, 0, st>>>(sums, q8_blocks(rows), cols, total, db, db_dtype);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}
