// Products of more rows with 4-bit weights, on the tensor cores with the weights in tensor memory.
//
// y[m][n] = sum over groups g of scale[n][g] (sum over the group's k of code[n][k] x[m][k]), as for few rows: codes are exact 16-bit floats, the
// inner sums are products of the tensor cores with 32-bit sums, and each group's is scaled and added in 32 bits. 128 rows of W
// are the instruction's rows. Four warps unpack their codes, a thread the 64 words of its row and block of 128
// columns, straight into tensor memory, from where the instruction takes them: in shared memory the tile would be written
// once and read once, which at these widths is more than shared memory gives. x lies there, at most 128 columns of
// it, laid out by asynchronous copies of three warps; a 32-bit x is three tiles of bfloat16 (its parts), three products into one sum. Eight
// warps take a group's sums out of tensor memory while the next group's are made, multiply them by their row's scale
// and keep the sums of up to 64 columns in registers. A cluster of up to 8 blocks shares the contraction where rows are
// few. Bound by what L2 delivers of x: each block reads all of it for its 128 rows.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "emr_act.h"
#include "emr_q4.h"
#include "emr_tc.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;

constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kUnpack = 4, kScale = 8, kLoad = 3;  // warps that unpack codes, scale sums and copy x; the last one issues
constexpr int kCodeStages = 6, kTileStages = 4, kMaxCluster = 8;
constexpr int kColumns = 512;                      // of tensor memory: two groups' sums of 128, then the tiles of codes, 64 each
constexpr int kRowPitch = 80;                      // of a row's 64 bytes of codes in shared memory: other banks than the row before

struct Params {
  const uint8_t* w;
  int64_t w_batch;
  int32_t tiles, blocks, row_blocks;
  int64_t N, K, M;
  const uint16_t* x;  // 16-bit values, `parts` matrices for each of x, `part` values apart
  int64_t x_batch, x_row, part;
  int32_t parts, half;  // half: float16
  int32_t step, width;  // columns of a block, and as the instruction has them: a multiple of 16
  int32_t stages;       // of x
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};

__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
      : "memory");
}
// 32 columns of a warp's 32 rows of tensor memory.
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
      "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
      "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
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

template <bool kHalf, int kPer>
__global__ void __launch_bounds__(kThreads, 1) q4_many_kernel(const __grid_constant__ Params p) {
  constexpr int kUnit = kQ4Codes + 32 * kPer, kCodeStage = 32 * kRowPitch;  // a warp's 32 rows are two units
  extern __shared__ __align__(16) uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kTileStages + 2 * 8 + 4];
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  const auto cluster = cg::this_cluster();
  const int shares = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const int x_part = p.width * 256, x_stage = p.parts * x_part;  // two tiles of 64 columns of W, 128 bytes a row, swizzled
  uint8_t* const ring = sm + p.stages * x_stage;
  // barriers: tiles of codes there and free, x there and free, sums there and free
  const uint32_t tile_full = smem_at(bars), tile_free = tile_full + 8 * kTileStages, x_full = tile_free + 8 * kTileStages, x_free = x_full + 64,
                 sum_full = x_free + 64, sum_free = sum_full + 16;
  volatile int* const stop = &gave_up;

  const unsigned here = blockIdx.x / unsigned(shares);
  const int64_t b = here / unsigned(p.row_blocks);
  const int block = int(here - unsigned(b) * unsigned(p.row_blocks));
  const int64_t m0 = int64_t(blockIdx.y) * p.step;
  const int columns = int(p.M - m0 < p.step ? p.M - m0 : p.step);
  const int first = int(unsigned(p.blocks) * unsigned(rank) / unsigned(shares)), last = int(unsigned(p.blocks) * unsigned(rank + 1) / unsigned(shares));

  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < kTileStages; i++) bar_init(tile_full + 8 * i, kUnpack), bar_init(tile_free + 8 * i, 1);
    for (int i = 0; i < p.stages; i++) bar_init(x_full + 8 * i, kLoad), bar_init(x_free + 8 * i, 1);
    for (int i = 0; i < 2; i++) bar_init(sum_full + 8 * i, 1), bar_init(sum_free + 8 * i, kScale);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWarps - 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_base)), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_base;

  float sum[4][16];
#pragma unroll
  for (int c = 0; c < 4; c++)
#pragma unroll
    for (int i = 0; i < 16; i++) sum[c][i] = 0.f;
  const int quarter = warp & 3;                                                    // rows of tensor memory that a warp may use
  const int chunks = p.width / 16, half = (chunks + 1) / 2, c0 = warp >= 8 ? half : 0;  // of 16 columns; a scaling warp's
  const int own = warp >= 8 ? chunks - half : half;

  if (warp < kUnpack) {
    const int tile = block * 8 + quarter * 2;
    const uint8_t* unit = p.w + b * p.w_batch + (int64_t(tile) * p.blocks + first) * kUnit + lane * 16;
    const int64_t second = int64_t(p.blocks) * kUnit;
    uint8_t* const codes_at = ring + warp * (kCodeStages * kCodeStage);
    const uint32_t to = smem_at(codes_at) + (lane >> 2) * kRowPitch + (lane & 3) * 16;
    const bool one = tile < p.tiles, two = tile + 1 < p.tiles;
    int put = 0;
    const auto issue = [&](int kb) {
      if (kb < last) {
        const uint32_t at = to + put * kCodeStage;
        if (one) copy16(at, unit), copy16(at + 8 * kRowPitch, unit + 512);
        if (two) copy16(at + 16 * kRowPitch, unit + second), copy16(at + 24 * kRowPitch, unit + second + 512);
        unit += kUnit;
        put = put == kCodeStages - 1 ? 0 : put + 1;
      }
      commit();
    };
    for (int i = 0; i < kCodeStages - 1; i++) issue(first + i);
    int get = 0;
    Ring<kTileStages> tiles;
    for (int kb = first; kb < last; kb++, tiles.next()) {
      issue(kb + kCodeStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kCodeStages - 1) : "memory");
      __syncwarp();
      uint4 c[4];
#pragma unroll
      for (int t = 0; t < 4; t++) c[t] = *reinterpret_cast<const uint4*>(codes_at + get * kCodeStage + lane * kRowPitch + t * 16);
      __syncwarp();
      get = get == kCodeStages - 1 ? 0 : get + 1;
      if (!warp_wait(tile_free + 8 * tiles.stage, tiles.round ^ 1, stop, 11)) break;
      fence_after();
      const uint32_t at = tmem + 256 + 64 * tiles.stage + (uint32_t(quarter * 32) << 16);
#pragma unroll
      for (int h = 0; h < 2; h++) {  // 64 columns of W
        uint32_t r[32];
#pragma unroll
        for (int v = 0; v < 2; v++)
#pragma unroll
          for (int t = 0; t < 4; t++) {
            const uint32_t w = (&c[t].x)[h * 2 + v];
#pragma unroll
            for (int j = 0; j < 4; j++) r[v * 16 + t * 4 + j] = codes<kHalf>(w >> (4 * j));
          }
        tmem_store32(at + h * 32, r);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(tile_full + 8 * tiles.stage);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp < kUnpack + kScale) {
    const int tile_row = quarter * 32 + lane, row = tile_row & 15, tile = block * 8 + (tile_row >> 4);
    const uint8_t* scales = p.w + b * p.w_batch + (int64_t(tile < p.tiles ? tile : 0) * p.blocks + first) * kUnit + q4_scale_at(row, 0, kQ4Cols / kPer);
    typedef std::conditional_t<kPer == 1, uint16_t, std::conditional_t<kPer == 2, uint32_t, uint2>> Word;
    Word next = __ldg(reinterpret_cast<const Word*>(scales));
    Ring<2> sums;
    bool ok = true;
    for (int kb = first; kb < last && ok; kb++) {
      const Word now = next;
      scales += kUnit;
      if (kb + 1 < last) next = __ldg(reinterpret_cast<const Word*>(scales));
#pragma unroll
      for (int q = 0; q < kPer; q++, sums.next()) {
        if (!(ok = warp_wait(sum_full + 8 * sums.stage, sums.round, stop, 12))) break;
        fence_after();
        const float scale = __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(&now)[q]) << 16);
        const uint32_t at = tmem + 128 * sums.stage + 16 * c0 + (uint32_t(quarter * 32) << 16);
#pragma unroll
        for (int c = 0; c < 4; c += 2) {  // as many as registers hold beside the sums
          uint32_t v[2][16];
          if (c < own) tmem_load16(at + 16 * c, v[0]);
          if (c + 1 < own) tmem_load16(at + 16 * c + 16, v[1]);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (c == 2) {
            fence_before();
            __syncwarp();
            if (lane == 0) arrive(sum_free + 8 * sums.stage);
          }
#pragma unroll
          for (int h = 0; h < 2; h++)
            if (c + h < own) {
#pragma unroll
              for (int i = 0; i < 16; i++) sum[c + h][i] = fmaf(scale, __uint_as_float(v[h][i]), sum[c + h][i]);
            }
        }
      }
    }
  } else if (warp < kWarps - 1) {
    // a thread has one 16-byte column of every sixth row
    const int id = threadIdx.x - 32 * (kUnpack + kScale), piece = id & 15, row0 = id >> 4;
    const int lag = p.stages > 3 ? 2 : 1;  // stages that a thread's copies are in flight
    const uint16_t* from = p.x + b * p.x_batch + (m0 + row0) * p.x_row + int64_t(first) * kQ4Cols + piece * 8;
    int64_t left = p.K - int64_t(first) * kQ4Cols - piece * 8;
    const uint32_t to = smem_at(sm) + (piece >> 3) * (p.width * 128);
    int put = 0, done = 0;
    uint32_t round = 0;
    bool ok = true;
    const auto ready = [&](int pending) {
      if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
      else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 0;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive(x_full + 8 * done);
      done = done == p.stages - 1 ? 0 : done + 1;
    };
    int in_flight = 0;
    for (int kb = first; kb < last; kb++) {
      if (!(ok = warp_wait(x_free + 8 * put, round ^ 1, stop, 13))) break;
      const int bytes = left >= 8 ? 16 : left > 0 ? int(left) * 2 : 0;
      for (int q = 0; q < p.parts; q++) {
        const uint16_t* source = from + q * p.part;
        uint32_t at = to + put * x_stage + q * x_part + row0 * 128;
        for (int m = row0; m < columns; m += 6, source += 6 * p.x_row, at += 6 * 128)
          copy16(at + (((piece & 7) ^ (m & 7)) << 4), bytes ? source : p.x, bytes);
      }
      commit();
      from += kQ4Cols, left -= kQ4Cols;
      if (++put == p.stages) put = 0, round ^= 1;
      if (++in_flight > lag) ready(lag), in_flight--;
    }
    if (ok)
      while (in_flight > 0) ready(--in_flight);
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    const uint32_t idesc = (1u << 4) | (kHalf ? 0u : (1u << 7) | (1u << 10)) | (uint32_t(p.width >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    Ring<kTileStages> tiles;
    Ring<2> sums;
    int stage = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int kb = first; kb < last && ok; kb++, tiles.next()) {
      if (!warp_wait(tile_full + 8 * tiles.stage, tiles.round, stop, 14) || !warp_wait(x_full + 8 * stage, round, stop, 15)) break;
      const uint32_t a = tmem + 256 + 64 * tiles.stage, x_at = smem_at(sm) + stage * x_stage;
#pragma unroll
      for (int q = 0; q < kPer; q++, sums.next()) {
        if (!(ok = warp_wait(sum_free + 8 * sums.stage, sums.round ^ 1, stop, 16))) break;
        fence_after();
        if (elect_one()) {
          for (int part = 0; part < p.parts; part++)
#pragma unroll
            for (int k = q * (8 / kPer); k < (q + 1) * (8 / kPer); k++)  // 16 columns of W
              mma(tmem + 128 * sums.stage, a + 8 * k, operand_desc(x_at + part * x_part + (k >> 2) * (p.width * 128)) + 2 * (k & 3), idesc,
                  part > 0 || k > q * (8 / kPer));
          mma_commit(sum_full + 8 * sums.stage);
          if (q == kPer - 1) {
            mma_commit(tile_free + 8 * tiles.stage);
            mma_commit(x_free + 8 * stage);
          }
        }
        __syncwarp();
      }
      if (++stage == p.stages) stage = 0, round ^= 1;
    }
  }
  if (*stop) settle();
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == kWarps - 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns) : "memory");
  }

  const auto finish = [&](int64_t n, int m, float v) {
    if (n >= p.N || m >= columns) return;
    float z[1] = {v}, d[1];
    if (p.bias) z[0] += p.bias[b * p.N + n];
    activate<1, false>(p.act, z, d);
    store_scalar(p.out, p.out_dtype, (b * p.M + m0 + m) * p.N + n, z[0]);
  };
  const bool scales_sums = warp >= kUnpack && warp < kUnpack + kScale;
  if (shares == 1) {
    if (scales_sums) {
      const int64_t n = int64_t(block) * 128 + quarter * 32 + lane;
      const float bias = p.bias && n < p.N ? p.bias[b * p.N + n] : 0.f;
      const int64_t at = (b * p.M + m0 + c0 * 16) * p.N + n;
#pragma unroll
      for (int c = 0; c < 4; c++) {
        if (c >= own || n >= p.N) break;
        float d[16];
#pragma unroll
        for (int i = 0; i < 16; i++) sum[c][i] += bias;
        activate<16, false>(p.act, sum[c], d);
#pragma unroll
        for (int i = 0; i < 16; i++)
          if ((c0 + c) * 16 + i < columns) store_scalar(p.out, p.out_dtype, at + int64_t(c * 16 + i) * p.N, sum[c][i]);
      }
    }
    return;
  }
  // the blocks' sums, [column][row], each block takes every so many columns
  float* const sums = reinterpret_cast<float*>(sm);
  if (scales_sums) {
#pragma unroll
    for (int c = 0; c < 4; c++)
      if (c < own) {
#pragma unroll
        for (int i = 0; i < 16; i++) sums[((c0 + c) * 16 + i) * 128 + quarter * 32 + lane] = sum[c][i];
      }
  }
  cluster.sync();
  for (int m = rank + (int(threadIdx.x) >> 7) * shares; m < columns; m += shares * (kThreads / 128)) {
    const int n = threadIdx.x & 127;
    float v = 0.f;
    for (int i = 0; i < shares; i++) v += cluster.map_shared_rank(sums, i)[m * 128 + n];
    finish(int64_t(block) * 128 + n, m, v);
  }
  cluster.sync();  // a block's sums are read by the others
}

// x as 16-bit values in rows of whole blocks, zero past K: what is not so already, and the parts of 32-bit values.
template <typename T>
__global__ void __launch_bounds__(256) q4_parts_kernel(const T* x, int64_t M, int64_t K, int64_t blocks, int64_t batch_stride, int64_t row_stride,
                                                       int64_t col_stride, int64_t total, uint16_t* out) {
  constexpr bool kSplit = sizeof(T) == 4;
  const int64_t quads = blocks * (kQ4Cols / 4), part = M * blocks * kQ4Cols;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {  // four columns
    const int64_t line = i / quads, k = (i - line * quads) * 4, b = line / M, m = line - b * M;
    const T* const from = x + b * batch_stride + m * row_stride + k * col_stride;
    T v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = k + j < K ? from[j * col_stride] : T(0.f);
    uint16_t* const to = out + b * (kSplit ? 3 : 1) * part + m * blocks * kQ4Cols + k;
    if constexpr (kSplit) {
      uint2 w[3];
      split_pair(v[0], v[1], w[0].x, w[1].x, w[2].x);
      split_pair(v[2], v[3], w[0].y, w[1].y, w[2].y);
#pragma unroll
      for (int q = 0; q < 3; q++) *reinterpret_cast<uint2*>(to + q * part) = w[q];
    } else {
      uint2 w;
      uint16_t* const e = reinterpret_cast<uint16_t*>(&w);
#pragma unroll
      for (int j = 0; j < 4; j++) e[j] = *reinterpret_cast<const uint16_t*>(v + j);
      *reinterpret_cast<uint2*>(to) = w;
    }
  }
}

template <bool kHalf, int kPer>
emr_status launch(const Params& p, int64_t blocks, int shares, int dev, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(q4_many_kernel<kHalf, kPer>, kMostSmem, dev, done)) return EMR_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(blocks * shares), unsigned((p.M + p.step - 1) / p.step));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kMostSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = unsigned(shares);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = shares > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, q4_many_kernel<kHalf, kPer>, p) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

}  // namespace

namespace emr {

emr_status q4_wait_error(int32_t* code, cudaStream_t st) { return take_wait_error(g_wait_error, code, st); }

size_t q4_many_room(const Q4Product& a) {
  if (a.dtype != EMR_F32 && a.whole) return 0;
  return size_t(a.x_batch) * (a.dtype == EMR_F32 ? 3 : 1) * size_t(a.rows) * size_t(q4_blocks(a.w->cols)) * kQ4Cols * 2;
}

emr_status launch_q4_many(const Q4Product& a, void* ws, int dev, int sms, cudaStream_t st) {
  Params p{};
  p.w = a.w->data, p.tiles = int32_t(q4_tiles(a.w->rows)), p.blocks = int32_t(q4_blocks(a.w->cols)), p.row_blocks = (p.tiles + 7) / 8;
  p.w_batch = a.w->batch == 1 ? 0 : int64_t(p.tiles) * p.blocks * q4_unit(a.w->group);
  p.N = a.w->rows, p.K = a.w->cols, p.M = a.rows;
  p.parts = a.dtype == EMR_F32 ? 3 : 1, p.half = a.dtype == EMR_F16;
  p.bias = a.bias, p.act = a.act, p.out = a.out, p.out_dtype = a.out_dtype;
  if (q4_many_room(a) == 0) {
    p.x = static_cast<const uint16_t*>(a.x), p.x_row = a.row_stride, p.x_batch = a.x_batch == 1 ? 0 : a.batch_stride;
  } else {
    const int64_t pitch = int64_t(p.blocks) * kQ4Cols, total = int64_t(a.x_batch) * a.rows * (pitch / 4);
    const int64_t wanted = (total + 255) / 256;
    const unsigned grid = unsigned(wanted < 16 * sms ? wanted : 16 * sms);
    uint16_t* const out = static_cast<uint16_t*>(ws);
    if (a.dtype == EMR_F32)
      q4_parts_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float*>(a.x), a.rows, p.K, p.blocks, a.batch_stride, a.row_stride, a.col_stride, total, out);
    else  // of both 16-bit types the bits are copied
      q4_parts_kernel<__half><<<grid, 256, 0, st>>>(static_cast<const __half*>(a.x), a.rows, p.K, p.blocks, a.batch_stride, a.row_stride, a.col_stride, total, out);
    if (cudaPeekAtLastError() != cudaSuccess) return EMR_ERR_CUDA;
    p.x = out, p.x_row = pitch, p.part = a.rows * pitch, p.x_batch = a.x_batch == 1 ? 0 : p.parts * p.part;
    p.K = pitch;
  }
  const int most = p.parts == 3 ? 64 : 128;
  const int64_t chunks = (p.M + most - 1) / most, batch = a.x_batch > a.w->batch ? a.x_batch : a.w->batch, blocks = batch * p.row_blocks;
  if (chunks > 65535 || blocks > INT32_MAX / kMaxCluster) return EMR_ERR_RANGE;
  p.step = int((p.M + chunks - 1) / chunks), p.width = (p.step + 15) / 16 * 16;
  int shares = 1;
  for (int s = 2; s <= kMaxCluster; s++)
    if (blocks * s * chunks <= sms && p.blocks / s >= 4) shares = s;
  const int room = kMostSmem - 1024 - kUnpack * kCodeStages * 32 * kRowPitch, stage = p.parts * p.width * 256;
  p.stages = room / stage < 8 ? room / stage : 8;
  const int per = kQ4Cols / a.w->group;
  if (p.half) return per == 1 ? launch<true, 1>(p, blocks, shares, dev, st) : per == 2 ? launch<true, 2>(p, blocks, shares, dev, st) : launch<true, 4>(p, blocks, shares, dev, st);
  return per == 1 ? launch<false, 1>(p, blocks, shares, dev, st) : per == 2 ? launch<false, 2>(p, blocks, shares, dev, st) : launch<false, 4>(p, blocks, shares, dev, st);
}

}  // namespace emr
