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

// Dense source: four columns c .. c + 3 of a row, zero past the matrix. kVector: columns
// are neighbours and every row is aligned to four elements.
template <typename T, bool kVector>
struct Dense {
  const T* p;
  int64_t batch_stride, row_stride, col_stride;
  __device__ __forceinline__ Four<T> four(const T* row, int64_t c, int64_t cols) const {
    Four<T> v;
    if (kVector && c + 4 <= cols) {
      v.load(row + c);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) v.set(j, c + j < cols ? row[(c + j) * (kVector ? 1 : col_stride)] : T(0.f));
    }
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
template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads) q8_rows_kernel(Dense<T, kVector> src, int64_t rows, int64_t cols, int64_t units,
                                                           emr_q8 q) {
  const int64_t chunks = q8_scale_chunks(cols), blocks = q8_blocks(cols), row_bytes = q8_row_bytes(cols);
  const int64_t unit = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (unit >= units) return;
  const int lane = threadIdx.x & 31;
  // divisions in 32 bits where they suffice: they cost as much as a block's work otherwise
  const bool small = units <= UINT32_MAX;
  const int64_t row = small ? uint32_t(unit) / uint32_t(chunks) : unit / chunks, chunk = unit - row * chunks;
  const int64_t b = small ? uint32_t(row) / uint32_t(rows) : row / rows, r = row - b * rows;
  const T* from = src.p + b * src.batch_stride + r * src.row_stride;
  const int64_t c = chunk * 512 + lane * 4;
  Four<T> u[4];
#pragma unroll
  for (int j = 0; j < 4; j++) u[j] = src.four(from, c + j * 128, cols);
  uint8_t* out = q.values + row * row_bytes + c;
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    float4 v = u[j].floats();
    const uint32_t byte = q8_warp_scale(v);
    word |= byte << (8 * j);
    if (chunk * 4 + j < blocks)
      *reinterpret_cast<uint32_t*>(out + j * 128) = q8_pack4(v.x, v.y, v.z, v.w, q8_inverse(byte));
  }
  if (lane == 0)
    *reinterpret_cast<uint32_t*>(q.scales + b * q8_scale_batch(rows, cols) + q8_scale_at(chunks, r, chunk * 4)) = word;
}

// One 128 x 128 tile: row blocks to q, column blocks (the transpose) to qt, column
// sums to sums[b][row tile][cols]. Mode 0: a dense source; 1: the values of an 8-bit
// matrix; 2: the product of a dense matrix and an 8-bit one. A warp has the rows
// 16 warp .. 16 warp + 15 and loads eight of them before it uses the first.
template <int kMode, typename T, bool kVector>
__global__ void __launch_bounds__(kThreads, 3) q8_tile_kernel(Dense<T, kVector> src, emr_q8 other, int64_t rows, int64_t cols,
                                                              emr_q8 q, emr_q8 qt, float* sums) {
  extern __shared__ float4 tile[];  // [128][32]
  __shared__ uint8_t row_scales[128], col_scales[128];
  const int64_t row_tiles = q8_blocks(rows), col_tiles = q8_blocks(cols);
  const int64_t ct = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles, rt = rest % row_tiles, b = rest / row_tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t chunks = q8_scale_chunks(cols), row_bytes = q8_row_bytes(cols), scale_batch = q8_scale_batch(rows, cols);
  const int64_t c = ct * 128 + lane * 4;
  const int64_t left = rows - rt * 128;
  const int have = int(left < 128 ? left : 128);  // rows of the tile
  const int wide = int(cols - ct * 128 < 128 ? cols - ct * 128 : 128);
  const int first = warp * 16;
  const T* from = kMode != 1 ? src.p + b * src.batch_stride + (rt * 128 + first) * src.row_stride : nullptr;
  const int64_t at = (b * rows + rt * 128 + first) * row_bytes + c;  // of the warp's first row in 8-bit matrices of this shape
  const uint8_t* codes = kMode != 0 ? other.values + at : nullptr;
  uint8_t* out = q.values ? q.values + at : nullptr;
  uint32_t scale_bytes = 127;
  if (kMode != 0 && lane < 16 && first + lane < have)
    scale_bytes = other.scales[b * scale_batch + q8_scale_at(chunks, rt * 128 + first + lane, ct)];
#pragma unroll
  for (int i0 = 0; i0 < 16; i0 += 8) {
    Four<T> u[8];
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (first + i0 + i < have) {
        if (kMode != 1) u[i] = src.four(from + (i0 + i) * src.row_stride, c, cols);
        if (kMode != 0) code[i] = *reinterpret_cast<const uint32_t*>(codes + (i0 + i) * row_bytes);
      }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int r = first + i0 + i;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < have) {
        if (kMode != 1) v = u[i].floats();
        if (kMode != 0) {
          const float s = q8_scale(__shfl_sync(0xffffffffu, scale_bytes, i0 + i));
          float4 d = q8_unpack4(code[i]);
          d = make_float4(d.x * s, d.y * s, d.z * s, d.w * s);
          // one rounding each, so that the values are those of the plain product
          v = kMode == 1 ? d : make_float4(__fmul_rn(v.x, d.x), __fmul_rn(v.y, d.y), __fmul_rn(v.z, d.z), __fmul_rn(v.w, d.w));
        }
      }
      tile[r * 32 + (lane ^ ((r >> 2) & 7))] = v;
      if (out && r < have) {
        const uint32_t byte = q8_warp_scale(v);
        *reinterpret_cast<uint32_t*>(out + (i0 + i) * row_bytes) = q8_pack4(v.x, v.y, v.z, v.w, q8_inverse(byte));
        if (lane == 0) row_scales[r] = uint8_t(byte);
      }
    }
  }
  __syncthreads();
  const int64_t t_row_bytes = q8_row_bytes(rows);
  uint8_t* tout = qt.values ? qt.values + (b * cols + ct * 128) * t_row_bytes + rt * 128 + lane * 4 : nullptr;
  for (int i = warp; i < 32; i += kWarps) {  // columns 4 i .. 4 i + 3, rows 4 lane .. 4 lane + 3
    float4 v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = tile[(lane * 4 + j) * 32 + (i ^ (lane & 7))];
    float4 col[4] = {make_float4(v[0].x, v[1].x, v[2].x, v[3].x), make_float4(v[0].y, v[1].y, v[2].y, v[3].y),
                     make_float4(v[0].z, v[1].z, v[2].z, v[3].z), make_float4(v[0].w, v[1].w, v[2].w, v[3].w)};
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const int n = i * 4 + j;
      if (sums) {
        float s = (col[j].x + col[j].y) + (col[j].z + col[j].w);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0 && n < wide) sums[(b * row_tiles + rt) * cols + ct * 128 + n] = s;
      }
      if (tout && n < wide) {
        const uint32_t byte = q8_warp_scale(col[j]);
        *reinterpret_cast<uint32_t*>(tout + n * t_row_bytes) = q8_pack4(col[j].x, col[j].y, col[j].z, col[j].w, q8_inverse(byte));
        if (lane == 0) col_scales[n] = uint8_t(byte);
      }
    }
  }
  __syncthreads();
  const int i = threadIdx.x;
  if (out && i < have) q.scales[b * scale_batch + q8_scale_at(chunks, rt * 128 + i, ct)] = row_scales[i];
  if (tout && i >= 128 && i - 128 < wide)
    qt.scales[b * q8_scale_batch(cols, rows) + q8_scale_at(q8_scale_chunks(rows), ct * 128 + i - 128, rt)] = col_scales[i - 128];
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

template <int kMode, typename T, bool kVector>
emr_status launch_tile(const Dense<T, kVector>& src, const emr_q8* other, int64_t batch, int64_t rows, int64_t cols,
                       const emr_q8* q, const emr_q8* qt, float* sums, cudaStream_t st) {
  const int64_t tiles = batch * q8_blocks(rows) * q8_blocks(cols);
  if (tiles > kMaxGrid) return EMR_ERR_RANGE;
  if (cudaFuncSetAttribute(q8_tile_kernel<kMode, T, kVector>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileBytes) != cudaSuccess)
    return EMR_ERR_CUDA;
  const emr_q8 none{};
  q8_tile_kernel<kMode, T, kVector><<<unsigned(tiles), kThreads, kTileBytes, st>>>(
      src, other ? *other : none, rows, cols, q ? *q : none, qt ? *qt : none, sums);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

template <typename T, bool kVector>
emr_status launch_rows(const Dense<T, kVector>& src, int64_t batch, int64_t rows, int64_t cols, const emr_q8* q, cudaStream_t st) {
  const int64_t units = batch * rows * q8_scale_chunks(cols), grid = (units + kWarps - 1) / kWarps;
  if (grid > kMaxGrid) return EMR_ERR_RANGE;
  q8_rows_kernel<T, kVector><<<unsigned(grid), kThreads, 0, st>>>(src, rows, cols, units, *q);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

struct DenseArgs {
  const void* p;
  int32_t dtype;
  int64_t batch, rows, cols, batch_stride, row_stride, col_stride;
};
template <typename Fn, typename T>
emr_status with_vector(const DenseArgs& a, Fn fn) {
  const bool vector = a.col_stride == 1 && reinterpret_cast<uintptr_t>(a.p) % (4 * sizeof(T)) == 0 &&
                      (a.rows == 1 || a.row_stride % 4 == 0) && (a.batch == 1 || a.batch_stride % 4 == 0);
  const T* p = static_cast<const T*>(a.p);
  return vector ? fn(Dense<T, true>{p, a.batch_stride, a.row_stride, a.col_stride})
                : fn(Dense<T, false>{p, a.batch_stride, a.row_stride, a.col_stride});
}
// fn with the source in its type, and as vectors where its layout allows.
template <typename Fn>
emr_status with_dense(const DenseArgs& a, Fn fn) {
  if (a.dtype == EMR_F32) return with_vector<Fn, float>(a, fn);
  if (a.dtype == EMR_BF16) return with_vector<Fn, __nv_bfloat16>(a, fn);
  return with_vector<Fn, __half>(a, fn);
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
  const DenseArgs args{src, dtype, batch, rows, cols, batch_stride, row_stride, col_stride};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_dense(args, [&](auto d) {
    return qt ? launch_tile<0>(d, nullptr, batch, rows, cols, q, qt, nullptr, st) : launch_rows(d, batch, rows, cols, q, st);
  });
}

extern "C" emr_status emr_q8_transpose(const emr_q8* q, const emr_q8* qt, void* stream) {
  if (!q8_ok(q) || !same_shape(qt, q->batch, q->cols, q->rows)) return EMR_ERR_ARG;
  return launch_tile<1>(Dense<float, true>{}, q, q->batch, q->rows, q->cols, nullptr, qt, nullptr,
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
  const DenseArgs args{dy, dtype, batch, rows, cols, rows * cols, cols, 1};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  float* sums = db ? static_cast<float*>(ws) : nullptr;
  const emr_status e = with_dense(args, [&](auto src) {
    return d ? launch_tile<2>(src, d, batch, rows, cols, dz, dzt, sums, st)
             : launch_tile<0>(src, nullptr, batch, rows, cols, dz, dzt, sums, st);
  });
  if (e != EMR_OK || !db) return e;
  const int64_t total = int64_t(batch) * cols, grid = (total + kThreads - 1) / kThreads;
  if (grid > kMaxGrid) return EMR_ERR_RANGE;
  q8_sums_kernel<<<unsigned(grid), kThreads, 0, st>>>(sums, q8_blocks(rows), cols, total, db, db_dtype);
  return cudaGetLastError() == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}
