// Products of a few rows with 4-bit weights: y = act(x W^T + b), as a layer that serves single patterns wants them.
//
// y[m][n] = sum over groups g of scale[n][g] (sum over the group's k of code[n][k] x[m][k]): the inner sums are m16n8k16
// instructions with 16 rows of W as the instruction's rows and rows of x as its 8 columns, exact products with sums in 32
// bits, and each is scaled and added in 32 bits. Codes become 16-bit floats by one OR and one subtraction for two (128 + q as bfloat16,
// 1024 + q as float16). A 32-bit x is three bfloat16 parts of 8 bits each, together all of its 24 bits, as
// three columns. Bound by reading W: half a byte an entry and 2 / group for its scale, once for up to 64 columns. A warp streams its
// units (16 rows x 128 columns, one piece of memory) into a ring of its own in shared memory by
// asynchronous copies, six units ahead; x lies in shared memory in the order in which lanes read it. The warps of a block share rows or
// the contraction; a cluster of up to 8 blocks shares the contraction of long rows and adds its parts through distributed shared memory in
// the order of blocks.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "emr_act.h"
#include "emr_q4.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;

constexpr int kThreads = 256, kWarps = kThreads / 32, kAhead = 6, kMaxCluster = 8;
constexpr int kRoomX = 32 * 1024;  // of x in shared memory at a time, twice that for more than 16 columns

struct Params {
  const uint8_t* w;
  int64_t w_batch;  // bytes of a matrix, 0 where all share it
  int32_t unit, tiles, blocks;
  int64_t N, K, M;
  const void* x;
  int64_t x_batch, x_row, x_col;
  int32_t x_vector;            // four columns are one aligned piece
  int32_t step;                // rows of x of a block
  int32_t wide;                // row tiles of a block, each `kR` tiles of 16
  int32_t chunk, pitch;        // blocks of x in shared memory at a time, and bytes of a column there
  int32_t row_blocks;          // blocks along the rows of W
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

template <bool kHalf>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (kHalf)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two codes, 16 bits apart, as 16-bit floats.
template <bool kHalf>
__device__ __forceinline__ uint32_t codes(uint32_t w) {
  uint32_t r;
  if (kHalf) {
    r = (w & 0x000f000fu) | 0x64006400u;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(0x64086408u));
  } else {
    r = (w & 0x000f000fu) | 0x43004300u;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(0x43084308u));
  }
  return r;
}
// The three parts of a 32-bit value, as bits of bfloat16: each takes the next 8 bits of its fraction. Infinities and NaN are
// the first part alone.
__device__ __forceinline__ void parts(float v, uint32_t (&p)[3]) {
  const uint32_t u = __float_as_uint(v);
  p[0] = u >> 16, p[1] = p[2] = 0;
  if ((u & 0x7f800000u) == 0x7f800000u) {
    if (u & 0x7fffffu) p[0] = 0x7fc0u;
    return;
  }
  const float left = v - __uint_as_float(u & 0xffff0000u);
  p[1] = __float_as_uint(left) >> 16;
  p[2] = __float_as_uint(left - __uint_as_float(__float_as_uint(left) & 0xffff0000u)) >> 16;
}

// T: x. kN: tiles of 8 columns. kPer: groups in 128 columns.
template <typename T, int kN, int kPer>
__global__ void __launch_bounds__(kThreads, kN <= 2 ? 3 : 1) q4_few_kernel(const __grid_constant__ Params p) {
  constexpr bool kSplit = sizeof(T) == 4, kHalf = std::is_same<T, __half>::value;
  constexpr int kR = kN >= 4 ? 2 : 1;  // tiles of 16 rows of a warp, which share what is read of x
  constexpr int kUnit = kQ4Codes + 32 * kPer, kStage = kR * kUnit;
  extern __shared__ __align__(16) uint8_t smem[];
  const auto cluster = cg::this_cluster();
  const int shares = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int wide = p.wide, teams = kWarps / wide, in_rows = warp % wide, team = warp / wide;
  const int64_t group = blockIdx.x / unsigned(shares);
  const int64_t b = group / p.row_blocks;
  const int tile = (int(group % p.row_blocks) * wide + in_rows) * kR;
  const int64_t m0 = int64_t(blockIdx.y) * p.step;
  const int rows = int(p.M - m0 < p.step ? p.M - m0 : p.step), columns = kSplit ? 3 * rows : rows;
  const int first = int(int64_t(p.blocks) * rank / shares), last = int(int64_t(p.blocks) * (rank + 1) / shares);

  uint8_t* const ring = smem + warp * (kAhead * kStage);
  uint8_t* const xs = smem + kWarps * kAhead * kStage;
  const uint32_t ring_at = uint32_t(__cvta_generic_to_shared(ring));
  const uint8_t* const w = p.w + b * p.w_batch + int64_t(tile) * p.blocks * kUnit;

  // unit after unit of the warp's share, each kR tiles
  const int own = first + team < last ? (last - first - team + teams - 1) / teams : 0;
  const int mine = tile < p.tiles ? own : 0;
  const auto fetch = [&](int i) {
    if (i < mine) {
      const int kb = first + team + i * teams;
      const uint32_t to = ring_at + i % kAhead * kStage;
#pragma unroll
      for (int r = 0; r < kR; r++) {
        if (r && tile + r >= p.tiles) break;
        const uint8_t* const from = w + (int64_t(r) * p.blocks + kb) * kUnit;
#pragma unroll
        for (int o = 0; o < kQ4Codes; o += 512) copy16(to + r * kUnit + o + lane * 16, from + o + lane * 16);
        if (lane < 2 * kPer) copy16(to + r * kUnit + kQ4Codes + lane * 16, from + kQ4Codes + lane * 16);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < kAhead - 1; i++) fetch(i);

  float sum[kR][kN][4];
#pragma unroll
  for (int r = 0; r < kR; r++)
#pragma unroll
    for (int n = 0; n < kN; n++)
#pragma unroll
      for (int j = 0; j < 4; j++) sum[r][n][j] = 0.f;

  const T* const x = static_cast<const T*>(p.x) + b * p.x_batch + m0 * p.x_row;
  int i = 0;
  for (int from = first; from < last; from += p.chunk) {
    const int size = last - from < p.chunk ? last - from : p.chunk;
    // x of the chunk: four columns a thread, [column of the instruction][block][two steps][t][step][4]
    __syncthreads();
    for (int at = threadIdx.x; at < rows * size * 32; at += kThreads) {
      const int q = at % (size * 32), m = at / (size * 32);
      const int64_t k = int64_t(from) * kQ4Cols + q * 4;
      Four<T> v;
      const T* const source = x + m * p.x_row + k * p.x_col;
      if (p.x_vector && k + 4 <= p.K) {
        v.u = *reinterpret_cast<const decltype(v.u)*>(source);
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++) v.set(j, k + j < p.K ? source[j * p.x_col] : T(0.f));
      }
      const int s = q >> 2 & 7;
      uint8_t* const to = xs + (q >> 5) * 256 + (s >> 1) * 64 + (q & 3) * 16 + (s & 1) * 8;
      if constexpr (kSplit) {
        uint32_t e[4][3];
        parts(v.u.x, e[0]), parts(v.u.y, e[1]), parts(v.u.z, e[2]), parts(v.u.w, e[3]);
#pragma unroll
        for (int c = 0; c < 3; c++) *reinterpret_cast<uint2*>(to + (c * rows + m) * p.pitch) = make_uint2(e[0][c] | e[1][c] << 16, e[2][c] | e[3][c] << 16);
      } else {
        *reinterpret_cast<uint2*>(to + m * p.pitch) = v.u;
      }
    }
    __syncthreads();
    for (; i < mine && first + team + i * teams < from + size; i++) {
      fetch(i + kAhead - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      __syncwarp();
      const uint8_t* const unit = ring + i % kAhead * kStage;
      const uint8_t* const x_at = xs + (first + team + i * teams - from) * 256 + t * 16 + g * p.pitch;
      uint4 code[kR][2];
      float scale[kR][2 * kPer];
#pragma unroll
      for (int r = 0; r < kR; r++) {
        code[r][0] = *reinterpret_cast<const uint4*>(unit + r * kUnit + lane * 16);
        code[r][1] = *reinterpret_cast<const uint4*>(unit + r * kUnit + 512 + lane * 16);
        uint32_t pair[kPer];
        const uint8_t* const at = unit + r * kUnit + kQ4Codes + g * 4 * kPer;
#pragma unroll
        for (int j = 0; j < kPer; j++) pair[j] = reinterpret_cast<const uint32_t*>(at)[j];
#pragma unroll
        for (int j = 0; j < 2 * kPer; j++) scale[r][j] = __uint_as_float(j & 1 ? pair[j >> 1] & 0xffff0000u : pair[j >> 1] << 16);
      }
#pragma unroll
      for (int c = 0; c < kPer; c++) {
        float part[kR][kN][4];
#pragma unroll
        for (int r = 0; r < kR; r++)
#pragma unroll
          for (int n = 0; n < kN; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) part[r][n][j] = 0.f;
#pragma unroll
        for (int v = c * (4 / kPer); v < (c + 1) * (4 / kPer); v++) {  // two steps
          uint32_t a[2][kR][4];
#pragma unroll
          for (int r = 0; r < kR; r++) {
            const uint32_t lo = (&code[r][0].x)[v], hi = (&code[r][1].x)[v];
#pragma unroll
            for (int h = 0; h < 2; h++) {
              a[h][r][0] = codes<kHalf>(lo >> (8 * h)), a[h][r][1] = codes<kHalf>(hi >> (8 * h));
              a[h][r][2] = codes<kHalf>(lo >> (8 * h + 4)), a[h][r][3] = codes<kHalf>(hi >> (8 * h + 4));
            }
          }
#pragma unroll
          for (int n = 0; n < kN; n++) {
            uint4 e = make_uint4(0, 0, 0, 0);
            if (n * 8 + g < columns) e = *reinterpret_cast<const uint4*>(x_at + v * 64 + n * 8 * p.pitch);
#pragma unroll
            for (int r = 0; r < kR; r++) {
              mma<kHalf>(part[r][n], a[0][r], e.x, e.y);
              mma<kHalf>(part[r][n], a[1][r], e.z, e.w);
            }
          }
        }
#pragma unroll
        for (int r = 0; r < kR; r++)
#pragma unroll
          for (int n = 0; n < kN; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) sum[r][n][j] = fmaf(scale[r][(j >> 1) * kPer + c], part[r][n][j], sum[r][n][j]);
      }
      __syncwarp();
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();

  // the warps' sums: [team][column][row of the block]; then those of the blocks of the cluster
  float* const sums = reinterpret_cast<float*>(smem);
  const int tall = wide * kR * 16, room = kN * 8 * tall;
#pragma unroll
  for (int r = 0; r < kR; r++)
#pragma unroll
    for (int n = 0; n < kN; n++)
#pragma unroll
      for (int j = 0; j < 4; j++)
        sums[team * room + (n * 8 + 2 * t + (j & 1)) * tall + (in_rows * kR + r) * 16 + g + 8 * (j >> 1)] = sum[r][n][j];
  __syncthreads();
  const int n0 = int(group % p.row_blocks) * tall;
  const int here = p.N - n0 < tall ? int(p.N - n0) : tall;
  const int outs = rows * tall;
  if (shares > 1) {
    for (int at = threadIdx.x; at < columns * tall; at += kThreads) {
      float v = sums[at];
      for (int i = 1; i < teams; i++) v += sums[i * room + at];
      sums[at] = v;
    }
    cluster.sync();
  }
  const int many = shares > 1 ? shares : teams;
  for (int at = threadIdx.x + (shares > 1 ? rank * kThreads : 0); at < outs; at += kThreads * (shares > 1 ? shares : 1)) {
    const int n = at % tall, m = at / tall;
    if (n >= here) continue;
    float z[1] = {0.f}, d[1];
    for (int c = 0; c < (kSplit ? 3 : 1); c++) {
      float part = 0.f;
      for (int i = 0; i < many; i++)
        part += shares > 1 ? cluster.map_shared_rank(sums, i)[c * outs + at] : sums[i * room + c * outs + at];
      z[0] += part;
    }
    if (p.bias) z[0] += p.bias[b * p.N + n0 + n];
    activate<1, false>(p.act, z, d);
    store_scalar(p.out, p.out_dtype, (b * p.M + m0 + m) * p.N + n0 + n, z[0]);
  }
  if (shares > 1) cluster.sync();  // a block's sums are read by the others
}

template <typename T, int kN, int kPer>
emr_status launch(const Params& p, int64_t blocks, int shares, size_t smem, int dev, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(q4_few_kernel<T, kN, kPer>, kMostSmem, dev, done)) return EMR_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(blocks * shares), unsigned((p.M + p.step - 1) / p.step));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = unsigned(shares);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = shares > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, q4_few_kernel<T, kN, kPer>, p) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

template <typename T, int kN>
emr_status launch(const Params& p, int per, int64_t blocks, int shares, size_t smem, int dev, cudaStream_t st) {
  return per == 1   ? launch<T, kN, 1>(p, blocks, shares, smem, dev, st)
         : per == 2 ? launch<T, kN, 2>(p, blocks, shares, smem, dev, st) : launch<T, kN, 4>(p, blocks, shares, smem, dev, st);
}

template <typename T>
emr_status plan(Params p, int64_t batch, int per, int dev, int sms, cudaStream_t st) {
  constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
  const int64_t most = 64 / kParts;
  const int64_t pieces = (p.M + most - 1) / most;
  p.step = int((p.M + pieces - 1) / pieces);
  const int columns = p.step * kParts, tiles8 = (columns + 7) / 8;
  const int kn = tiles8 <= 1 ? 1 : tiles8 <= 2 ? 2 : tiles8 <= 4 ? 4 : 8, kr = kn >= 4 ? 2 : 1;
  // Rows of a block: x is read by every block, so that its bytes should stay a quarter of the weights'
  int wide = 1;
  while (wide < kWarps && int64_t(p.step) * int(sizeof(T)) * 4 > int64_t(wide) * kr * 8) wide *= 2;
  while (wide > 1 && (p.tiles + wide * kr - 1) / (wide * kr) * batch < sms / 4) wide /= 2;
  p.wide = wide;
  p.row_blocks = (p.tiles + wide * kr - 1) / (wide * kr);
  const int64_t blocks = batch * p.row_blocks;
  int shares = 1;
  for (int s = 2; s <= kMaxCluster; s++)
    if (blocks * s <= 2 * sms && p.blocks / s >= 2 * (kWarps / wide)) shares = s;
  const int share = (p.blocks + shares - 1) / shares;
  int chunk = (kn > 2 ? 2 : 1) * kRoomX / (columns * 256);
  chunk = chunk < 1 ? 1 : chunk > share ? share : chunk;
  p.chunk = chunk, p.pitch = chunk * 256 + 64;
  const size_t ring = size_t(kWarps) * kAhead * kr * p.unit, sums = size_t(kWarps) * kr * 16 * kn * 8 * 4;
  size_t smem = ring + size_t(columns) * p.pitch;
  if (smem < sums) smem = sums;
  if (blocks * shares > INT32_MAX || (p.M + p.step - 1) / p.step > 65535) return EMR_ERR_RANGE;
  return kn == 1   ? launch<T, 1>(p, per, blocks, shares, smem, dev, st)
         : kn == 2 ? launch<T, 2>(p, per, blocks, shares, smem, dev, st)
         : kn == 4 ? launch<T, 4>(p, per, blocks, shares, smem, dev, st) : launch<T, 8>(p, per, blocks, shares, smem, dev, st);
}

}  // namespace

extern "C" emr_status emr_q4_matmul(const void* x, int32_t dtype, int32_t x_batch, int64_t rows, int64_t batch_stride, int64_t row_stride,
                                    int64_t col_stride, const emr_q4* w, const float* bias, int32_t act, void* out, int32_t out_dtype,
                                    void* stream) {
  if (!q4_ok(w) || !x || !out || rows < 1 || x_batch < 1 || (x_batch != 1 && w->batch != 1 && x_batch != w->batch) || !dtype_ok(dtype) ||
      !dtype_ok(out_dtype) || batch_stride < 0 || row_stride < 0 || col_stride < 0 || act < EMR_ACT_IDENTITY || act > EMR_ACT_ABS ||
      reinterpret_cast<uintptr_t>(x) % dtype_bytes(dtype) || reinterpret_cast<uintptr_t>(out) % dtype_bytes(out_dtype) ||
      reinterpret_cast<uintptr_t>(bias) % 4)
    return EMR_ERR_ARG;
  size_t bytes;
  const emr_status ok = emr_q4_size(w->batch, w->rows, w->cols, w->group, &bytes);
  if (ok != EMR_OK) return ok;
  if (rows > kQ8MaxDim) return EMR_ERR_RANGE;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Params p{};
  p.w = w->data, p.unit = q4_unit(w->group), p.tiles = int32_t(q4_tiles(w->rows)), p.blocks = int32_t(q4_blocks(w->cols));
  p.w_batch = w->batch == 1 ? 0 : int64_t(p.tiles) * p.blocks * p.unit;
  p.N = w->rows, p.K = w->cols, p.M = rows;
  p.x = x, p.x_batch = x_batch == 1 ? 0 : batch_stride, p.x_row = row_stride, p.x_col = col_stride;
  const int64_t batch = x_batch > w->batch ? x_batch : w->batch;
  const int piece = 4 * dtype_bytes(dtype);
  p.x_vector = col_stride == 1 && reinterpret_cast<uintptr_t>(x) % piece == 0 && (rows == 1 || row_stride % 4 == 0) &&
               (x_batch == 1 || batch_stride % 4 == 0);
  p.bias = bias, p.act = act, p.out = out, p.out_dtype = out_dtype;
  const int per = kQ4Cols / w->group;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == EMR_F32) return plan<float>(p, batch, per, dev, sms, st);
  if (dtype == EMR_BF16) return plan<__nv_bfloat16>(p, batch, per, dev, sms, st);
  return plan<__half>(p, batch, per, dev, sms, st);
}
