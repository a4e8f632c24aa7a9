// The product of a few rows (at most 8, 8192 values in all) with a small 8-bit weight matrix in
// one launch: a single answer, where a launch of its own to quantise x would cost as much as the
// product. Every block quantises x by itself. A warp takes 16 outputs and a share of the
// contraction, straight from memory into the registers of m16n8k32 instructions, whose 8 columns
// are the rows of x. The order within a block of 128 is the same for both operands but its own: a
// lane's 16 bytes feed two instructions, so that every load is 16 bytes a lane and a row's 64
// bytes are one piece. The sum of a block is scaled and added in 32 bits, the warps' shares
// are added in their order. What bounds it is latency: the wait for x, its quantising, and, as
// weights grow, the loads that a warp has in flight. Its time and that of the two launches of
// quantising and emr_q8_matmul, in a captured graph with the weights in L2 (us; few_fused is the rule):
//   rows  columns   1 MB         4 MB         8 MB         16 MB of weights
//   1     64        4.1   5.4    5.0   6.1    7.8   7.4    11.5   9.2
//   1     1024      2.7   6.4    3.9   6.6    6.2   7.2     6.7   8.2
//   2     4096      6.2   6.8    6.2   7.2    6.4   7.6     8.2   8.7
//   4     256       4.1   5.6    5.0   5.6    7.4   6.5    12.3   8.2
//   8     1024      5.0   6.4    6.2   6.7    9.9   7.2    14.5   8.0
//   16    256       8.8   6.0    9.5   6.0   17.2   7.0    29.5   9.0
// 5460 x 1364 with one row takes 4.5, and 7.2 by two launches.
#include <cuda_runtime.h>

#include "emr_act.h"
#include "emr_q8.h"

namespace {

using namespace emr;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Params {
  const uint8_t *w, *w_scales;
  int32_t N, w_one, x_one;
  int32_t M, K, blocks, chunks;  // columns, blocks of 128 of them, and scale chunks
  int32_t shares, groups;        // warps of a block that split the contraction; groups of 16 outputs
  const void* source;            // x
  int64_t batch_stride, row_stride, col_stride;
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// v * 2^(a - 127) * 2^(b - 127) for two scale bytes, in two steps of half the exponent each, so
// that neither overflows where the result does not.
__device__ __forceinline__ float scaled(float v, int a, int b) {
  const int e = a + b - 254, h = e >> 1;
  return v * __int_as_float((h + 127) << 23) * __int_as_float((e - h + 127) << 23);
}

__device__ __forceinline__ uint4 stream16(const uint8_t* p) {  // weights are read once
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

constexpr int kRows = 8;

template <typename T>
__global__ void __launch_bounds__(kThreads) q8_few_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) uint8_t codes[];  // [share][row][its blocks of 128, and 64 bytes]
  __shared__ float sums[kWarps][kRows][16];
  __shared__ uint8_t scales[64][kRows];  // [block][row]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int share = warp % p.shares, teams = kWarps / p.shares, team = warp / p.shares;
  const int b = blockIdx.y;
  const int group = blockIdx.x * teams + team;
  const int first = p.blocks * share / p.shares, last = p.blocks * (share + 1) / p.shares;
  const int64_t row_bytes = int64_t(p.blocks) * 128;
  const int g = lane >> 2, t = lane & 3;

  // x first when it comes from its source: the blocks of a share belong to the first team's warp
  const int pitch = ((p.blocks + p.shares - 1) / p.shares) * 128 + 64;
  uint8_t* const own = codes + share * p.M * pitch;
  grid_wait();
  grid_go();
  {
    if (team == 0) {
      const T* src = static_cast<const T*>(p.source) + (p.x_one ? 0 : b * p.batch_stride);
      for (int m = 0; m < p.M; m++)
        for (int kb = first; kb < last; kb++) {
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          {
            const int64_t c = kb * 128 + lane * 4;
            const T* at = src + m * p.row_stride + c * p.col_stride;
            if (c < p.K) v.x = float(at[0]);
            if (c + 1 < p.K) v.y = float(at[p.col_stride]);
            if (c + 2 < p.K) v.z = float(at[2 * p.col_stride]);
            if (c + 3 < p.K) v.w = float(at[3 * p.col_stride]);
          }
          const uint32_t byte = q8_warp_scale(v);
          *reinterpret_cast<uint32_t*>(own + m * pitch + (kb - first) * 128 + lane * 4) = q8_pack4(v.x, v.y, v.z, v.w, q8_inverse(byte));
          if (lane == 0) scales[kb][m] = uint8_t(byte);
        }
    }
    __syncthreads();
  }

  float acc[4] = {};
  if (group < p.groups) {
    const int r0 = min(group * 16 + g, p.N - 1), r1 = min(group * 16 + g + 8, p.N - 1);
    const int64_t wb = p.w_one ? 0 : b;
    const uint8_t* w = p.w + wb * p.N * row_bytes + t * 16;
    const uint8_t *w0 = w + r0 * row_bytes, *w1 = w + r1 * row_bytes;
    const uint8_t* ws = p.w_scales + wb * q8_scale_batch(p.N, int64_t(p.blocks) * 128);
    const uint8_t *s0 = ws + q8_scale_at(p.chunks, r0, 0), *s1 = ws + q8_scale_at(p.chunks, r1, 0);
    const int m = min(g, p.M - 1), m0 = min(2 * t, p.M - 1), m1 = min(2 * t + 1, p.M - 1);  // rows past M repeat the last; they are not stored
#pragma unroll 2
    for (int kb = first; kb < last; kb++) {
      const int64_t k = int64_t(kb) * 128;
      uint4 a[2][2], xv[2];
#pragma unroll
      for (int j = 0; j < 2; j++) a[0][j] = stream16(w0 + k + j * 64), a[1][j] = stream16(w1 + k + j * 64);
      const int at = (kb >> 2) * 512 + (kb & 3);
      const int sw0 = s0[at], sw1 = s1[at];
#pragma unroll
      for (int j = 0; j < 2; j++) xv[j] = *reinterpret_cast<const uint4*>(own + m * pitch + (kb - first) * 128 + j * 64 + t * 16);
      const int sx0 = scales[kb][m0], sx1 = scales[kb][m1];
      float c[4] = {};
#pragma unroll
      for (int j = 0; j < 2; j++) {
        mma(c, a[0][j].x, a[1][j].x, a[0][j].y, a[1][j].y, xv[j].x, xv[j].y);
        mma(c, a[0][j].z, a[1][j].z, a[0][j].w, a[1][j].w, xv[j].z, xv[j].w);
      }
      acc[0] += scaled(c[0], sw0, sx0), acc[1] += scaled(c[1], sw0, sx1);
      acc[2] += scaled(c[2], sw1, sx0), acc[3] += scaled(c[3], sw1, sx1);
    }
  }
  sums[warp][2 * t][g] = acc[0], sums[warp][2 * t + 1][g] = acc[1];
  sums[warp][2 * t][g + 8] = acc[2], sums[warp][2 * t + 1][g + 8] = acc[3];
  __syncthreads();
  for (int i = threadIdx.x; i < teams * kRows * 16; i += kThreads) {
    const int r = i & 15, m = i / 16 % kRows, tm = i / (16 * kRows);
    const int n = (blockIdx.x * teams + tm) * 16 + r;
    if (m >= p.M || n >= p.N) continue;
    float z[1] = {0.f}, d[1];
    for (int s = 0; s < p.shares; s++) z[0] += sums[tm * p.shares + s][m][r];
    if (p.bias) z[0] += p.bias[int64_t(b) * p.N + n];
    activate<1, false>(p.act, z, d);
    store_scalar(p.out, p.out_dtype, (int64_t(b) * p.M + m) * p.N + n, z[0]);
  }
}

template <typename T>
emr_status launch(const Params& p, int batch, cudaStream_t st) {
  const int teams = kWarps / p.shares;
  const size_t smem = size_t(p.shares) * p.M * (((p.blocks + p.shares - 1) / p.shares) * 128 + 64);
  return launch_after(q8_few_kernel<T>, dim3(unsigned((p.groups + teams - 1) / teams), unsigned(batch)), kThreads, smem, st, p);
}

}  // namespace

namespace emr {

emr_status launch_few(const FewArgs& a, cudaStream_t st) {
  Params p{};
  p.w = a.w->values, p.w_scales = a.w->scales, p.N = int32_t(a.w->rows), p.w_one = a.w->batch == 1;
  p.K = int32_t(a.w->cols), p.blocks = int32_t(q8_blocks(a.w->cols)), p.chunks = int32_t(q8_scale_chunks(a.w->cols));
  p.bias = a.bias, p.act = a.act, p.out = a.out, p.out_dtype = a.out_dtype;
  p.groups = (p.N + 15) / 16;
  // 16 warps for each of 152 SMs, as far as the contraction can be shared
  p.shares = 1;
  while (p.shares < kWarps && p.shares * 2 <= p.blocks && int64_t(p.groups) * a.batch * p.shares < 16 * 152) p.shares *= 2;
  p.M = int32_t(a.x_rows), p.x_one = a.x_batch == 1, p.source = a.x;
  p.batch_stride = a.x_batch_stride, p.row_stride = a.x_row_stride, p.col_stride = a.x_col_stride;
  if (a.x_dtype == EMR_F32) return launch<float>(p, a.batch, st);
  if (a.x_dtype == EMR_BF16) return launch<__nv_bfloat16>(p, a.batch, st);
  return launch<__half>(p, a.batch, st);
}

}  // namespace emr
