// Products of more rows with 4-bit weights, on the tensor cores with the weights in tensor memory.
//
// y[m][n] = sum over groups g of scale[n][g] (sum over the group's k of code[n][k] x[m][k]), as for few rows: codes are exact 16-bit floats, the
// inner sums are products of the tensor cores with 32-bit sums, and each group's is scaled and added in 32 bits. 128 rows of W
// are the instruction's rows. Four warps unpack their codes, a thread the 64 words of its row and block of 128
// columns, straight into tensor memory, from where the instruction takes them: in shared memory the tile would be written
// once and read once, which at these widths is more than shared memory gives. x, up to 128 rows of it, is laid out beforehand as
// its tiles lie in shared memory, so that one copy brings a block of columns; a 32-bit x is three tiles of bfloat16 (its parts), three
// products into one sum. Eight warps take a group's sums out of tensor memory while the next group's are made, multiply them by
// their row's scale and keep the sums of up to 64 columns in registers. A cluster of up to 8 blocks shares the contraction
// where rows are few. 101 x 16384 x 8192 bfloat16 takes 44 us, 8.5 of them beside the loop, which takes 1040 clocks a block of 128
// columns: the matrix pipe 450-570, a scaling warp 720, an unpacking warp 600, coupled by two buffers of sums. With 8 warps that
// unpack (96 registers a thread, and the sums spilled) it took 54; with 16 that scale (72) 79; with three buffers of sums and
// two of codes 48. Neither x (a fourteenth of it copied: 44) nor the multiplications (a quarter of them: 43) hold it.
// That is with groups of 128; a hand-over of sums for each 64 columns makes it 55, for each 32 96 (40 rows: 38, 51 and 92), and float32, two blocks of rows of three
// products each, 113, 143 and 239 (40 rows: 53, 73 and 122).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "emr_act.h"
#include "emr_q4.h"
#include "emr_tc.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;

constexpr int kUnpack = 4, kScale = 8;  // warps that unpack codes and scale sums; then one that copies x and one that issues
constexpr int kSums = 32 / kScale;  // 16 columns each of a scaling warp's sums
constexpr int kWarps = kUnpack + kScale + 2, kThreads = 32 * kWarps;
constexpr int kCodeStages = 8, kTileStages = 4, kMaxCluster = 8;
constexpr int kBatch = 512;              // bytes of scales that a warp has copied at a time, of 1024 / group blocks of columns
constexpr int kColumns = 512;            // of tensor memory: two groups' sums of 128, then the tiles of codes, 64 each
constexpr int kRowPitch = 80;            // of a row's 64 bytes of codes in shared memory: other banks than the row before

struct Params {
  const uint8_t* w;
  int64_t w_batch;
  int32_t tiles, blocks, row_blocks;
  int64_t N, K, M;
  const uint8_t* x;     // tiles of a block of columns after the other, those of `step` rows of x after the other
  int64_t x_batch;      // bytes of a matrix, 0 where all share it
  int32_t parts;        // tiles of a block: 1, or the 3 parts of 32-bit values
  int32_t step, width;  // rows of x of a block, and as the instruction has them: a multiple of 16
  int32_t stages;       // of x and of unpacked codes
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};

__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
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
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
// Two sums, two values at a time.
__device__ __forceinline__ void add_scaled(float& s0, float& s1, float scale, uint32_t v0, uint32_t v1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %2};\n\tmov.b64 b, {%3, %4};\n\tmov.b64 c, {%0, %1};\n\tfma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "+f"(s0), "+f"(s1) : "f"(scale), "r"(v0), "r"(v1));
}

template <bool kHalf, int kPer>
__global__ void __launch_bounds__(kThreads, 1) q4_many_kernel(const __grid_constant__ Params p) {
  constexpr int kUnit = kQ4Codes + 32 * kPer, kCodeStage = 32 * kRowPitch;  // a warp's 32 rows are two units
  extern __shared__ __align__(16) uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kTileStages + 4];
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  const auto cluster = cg::this_cluster();
  const int shares = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const int x_part = p.width * 256, x_stage = p.parts * x_part;  // two tiles of 64 columns of W, 128 bytes a row, swizzled
  uint8_t* const ring = sm + p.stages * x_stage;
  // barriers: x and unpacked codes there and free, sums there and free
  const uint32_t full = smem_at(bars), free_again = full + 8 * kTileStages, sum_full = free_again + 8 * kTileStages, sum_free = sum_full + 16;
  volatile int* const stop = &gave_up;

  const unsigned here = blockIdx.x / unsigned(shares);
  const int64_t b = here / unsigned(p.row_blocks);
  const int block = int(here - unsigned(b) * unsigned(p.row_blocks));
  const int64_t m0 = int64_t(blockIdx.y) * p.step;
  const int columns = int(p.M - m0 < p.step ? p.M - m0 : p.step);
  const int first = int(unsigned(p.blocks) * unsigned(rank) / unsigned(shares)), last = int(unsigned(p.blocks) * unsigned(rank + 1) / unsigned(shares));

  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < kTileStages; i++) bar_init(full + 8 * i, 4 + 1), bar_init(free_again + 8 * i, 1);
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

  const int quarter = warp & 3;                         // rows of tensor memory that a warp may use
  const int chunks = p.width / 16, each = (chunks + kScale / 4 - 1) / (kScale / 4);  // of 16 columns, and a scaling warp's
  const int c0 = (warp - kUnpack) / 4 * each, own = chunks - c0 < each ? chunks - c0 : each;

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
#pragma unroll 1
    for (int i = 0; i < kCodeStages - 1; i++) issue(first + i);
    int get = 0, stage = 0;
    uint32_t round = 0;
    for (int kb = first; kb < last; kb++) {
      issue(kb + kCodeStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kCodeStages - 1) : "memory");
      __syncwarp();
      uint4 c[4];
#pragma unroll
      for (int t = 0; t < 4; t++) c[t] = *reinterpret_cast<const uint4*>(codes_at + get * kCodeStage + lane * kRowPitch + t * 16);
      __syncwarp();
      get = get == kCodeStages - 1 ? 0 : get + 1;
      if (!warp_wait(free_again + 8 * stage, round ^ 1, stop, 11)) break;
      fence_after();
      const uint32_t at = tmem + 256 + 64 * stage + (uint32_t(quarter * 32) << 16);
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
      if (lane == 0) arrive(full + 8 * stage);
      if (++stage == p.stages) stage = 0, round ^= 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp < kUnpack + kScale) {
    float sum[kSums][16];  // alive in this branch alone: for all warps they would be spilled
#pragma unroll
    for (int c = 0; c < kSums; c++)
#pragma unroll
      for (int i = 0; i < 16; i++) sum[c][i] = 0.f;
    // the scales of its 32 rows, two units, of a batch of blocks while the batch before is used
    constexpr int kBlocks = 8 / kPer, kPieces = 4 * kPer;
    const int tile = block * 8 + quarter * 2, piece = lane % kPieces;
    const bool copies = tile + piece / (2 * kPer) < p.tiles;
    int ahead = first + lane / kPieces;
    const uint8_t* from = p.w + b * p.w_batch + ((int64_t(tile) + piece / (2 * kPer)) * p.blocks + ahead) * kUnit + kQ4Codes + piece % (2 * kPer) * 16;
    uint8_t* const scales = ring + kUnpack * kCodeStages * kCodeStage + (warp - kUnpack) * (2 * kBatch);
    uint32_t to = smem_at(scales) + lane * 16;
    const auto issue = [&]() {
      if (copies && ahead < last) copy16(to, from);
      ahead += kBlocks, from += kBlocks * kUnit, to ^= kBatch;
    };
    issue();
    const uint8_t* const mine = scales + (lane >> 4) * (32 * kPer) + (q4_scale_at(lane & 15, 0, kQ4Cols / kPer) - kQ4Codes);
    typedef std::conditional_t<kPer == 1, uint16_t, std::conditional_t<kPer == 2, uint32_t, uint2>> Word;
    Ring<2> sums;
    bool ok = true;
    int in_batch = 0, half = 0;
    for (int kb = first; kb < last && ok; kb++) {
      if (in_batch == 0) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        issue();
      }
      const Word now = *reinterpret_cast<const Word*>(mine + half + in_batch * (64 * kPer));
      if (++in_batch == kBlocks) in_batch = 0, half ^= kBatch;
#pragma unroll
      for (int q = 0; q < kPer; q++, sums.next()) {
        if (!(ok = warp_wait(sum_full + 8 * sums.stage, sums.round, stop, 12))) break;
        fence_after();
        const float scale = __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(&now)[q]) << 16);
        const uint32_t at = tmem + 128 * sums.stage + 16 * c0 + (uint32_t(quarter * 32) << 16);
        // 32 columns at a time
#pragma unroll
        for (int c = 0; c < kSums; c += 2) {
          uint32_t v[2][16];
          if (c < own) tmem_load16(at + 16 * c, v[0]);
          if (c + 1 < own) tmem_load16(at + 16 * c + 16, v[1]);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (c + 2 >= kSums) {
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(sum_free + 8 * sums.stage);
          }
#pragma unroll
          for (int h = 0; h < 2; h++)
            if (c + h < own) {
#pragma unroll
              for (int i = 0; i < 16; i += 2) add_scaled(sum[c + h][i], sum[c + h][i + 1], scale, v[h][i], v[h][i + 1]);
            }
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (shares == 1) {
      const int64_t n = int64_t(block) * 128 + quarter * 32 + lane;
      const float bias = p.bias && n < p.N ? p.bias[b * p.N + n] : 0.f;
      const int64_t at = (b * p.M + m0 + c0 * 16) * p.N + n;
#pragma unroll
      for (int c = 0; c < kSums; c++) {
        if (c >= own || n >= p.N) break;
        float d[16];
#pragma unroll
        for (int i = 0; i < 16; i++) sum[c][i] = (c0 + c) * 16 + i < columns ? sum[c][i] + bias : 0.f;  // x's tile holds anything there, and sin's way is one for all 16
        activate<16, false>(p.act, sum[c], d);
#pragma unroll
        for (int i = 0; i < 16; i++)
          if ((c0 + c) * 16 + i < columns) store_scalar(p.out, p.out_dtype, at + int64_t(c * 16 + i) * p.N, sum[c][i]);
      }
    } else {
      // for the cluster, [column][row], over x: the last of the sums was there after the last product
      float* const to_all = reinterpret_cast<float*>(sm);
#pragma unroll
      for (int c = 0; c < kSums; c++)
        if (c < own) {
#pragma unroll
          for (int i = 0; i < 16; i++) to_all[((c0 + c) * 16 + i) * 128 + quarter * 32 + lane] = sum[c][i];
        }
    }
  } else if (warp == kWarps - 2) {
    grid_wait();  // x has been laid out
    const uint8_t* from = p.x + b * p.x_batch + (int64_t(blockIdx.y) * p.blocks + first) * x_stage;
    uint32_t round = 0;
    int stage = 0;
    for (int kb = first; kb < last; kb++, from += x_stage) {
      if (!warp_wait(free_again + 8 * stage, round ^ 1, stop, 13)) break;
      if (elect_one()) {
        bar_expect(full + 8 * stage, uint32_t(x_stage));
        bulk_load(smem_at(sm) + stage * x_stage, from, uint32_t(x_stage), full + 8 * stage);
      }
      __syncwarp();
      if (++stage == p.stages) stage = 0, round ^= 1;
    }
  } else {
    const uint32_t idesc = (1u << 4) | (kHalf ? 0u : (1u << 7) | (1u << 10)) | (uint32_t(p.width >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    Ring<2> sums;
    uint32_t round = 0;
    int stage = 0;
    bool ok = true;
    for (int kb = first; kb < last && ok; kb++) {
      if (!warp_wait(full + 8 * stage, round, stop, 14)) break;
      const uint32_t a = tmem + 256 + 64 * stage, x_at = smem_at(sm) + stage * x_stage;
#pragma unroll
      for (int q = 0; q < kPer; q++, sums.next()) {
        if (!(ok = warp_wait(sum_free + 8 * sums.stage, sums.round ^ 1, stop, 15))) break;
        fence_after();
        const uint32_t d = tmem + 128 * sums.stage;
        for (int part = 0; part < p.parts; part++) {  // by the whole warp, as is all but the instructions
          const uint64_t x0 = operand_desc(x_at + part * x_part), x1 = operand_desc(x_at + part * x_part + p.width * 128);
          if (elect_one()) {
#pragma unroll
            for (int k = q * (8 / kPer); k < (q + 1) * (8 / kPer); k++)  // 16 columns of W
              mma(d, a + 8 * k, (k < 4 ? x0 : x1) + 2 * (k & 3), idesc, part > 0 || k > q * (8 / kPer));
          }
          __syncwarp();
        }
        if (elect_one()) {
          mma_commit(sum_full + 8 * sums.stage);
          if (q == kPer - 1) mma_commit(free_again + 8 * stage);
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
  if (shares == 1) return;
  const float* const sums = reinterpret_cast<const float*>(sm);
  cluster.sync();  // each block takes every so many columns
  for (int m = rank + (int(threadIdx.x) >> 7) * shares; m < columns && threadIdx.x < kThreads / 128 * 128; m += shares * (kThreads / 128)) {
    const int n = threadIdx.x & 127;
    float v = 0.f;
    for (int i = 0; i < shares; i++) v += cluster.map_shared_rank(sums, i)[m * 128 + n];
    finish(int64_t(block) * 128 + n, m, v);
  }
  cluster.sync();  // a block's sums are read by the others
}

// x as the tiles of the product's blocks: a thread's 8 columns of W, as they lie or one by one.
template <typename T>
__global__ void __launch_bounds__(256) q4_tiles_kernel(const T* x, int64_t M, int64_t K, int32_t blocks, int64_t batch_stride, int64_t row_stride,
                                                       int64_t col_stride, int32_t whole, int32_t step, int32_t width, int32_t chunks, int64_t total,
                                                       uint8_t* out) {
  constexpr bool kSplit = sizeof(T) == 4;
  constexpr int kParts = kSplit ? 3 : 1;
  grid_go();
  const int64_t pieces = int64_t(blocks) * 16;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
    const int64_t line = i / pieces, k = (i - line * pieces) * 8, b = line / M, m = line - b * M;
    const T* const from = x + b * batch_stride + m * row_stride + k * col_stride;
    uint32_t v[8];  // bits
    if (whole && k + 8 <= K) {
      const uint4 u = *reinterpret_cast<const uint4*>(from);
      v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
      if (kSplit) {
        const uint4 w = *reinterpret_cast<const uint4*>(from + 4);
        v[4] = w.x, v[5] = w.y, v[6] = w.z, v[7] = w.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const T e = k + j < K ? from[j * col_stride] : T(0.f);
        if constexpr (kSplit) v[j] = __float_as_uint(e);
        else if (j & 1) v[j >> 1] |= uint32_t(*reinterpret_cast<const uint16_t*>(&e)) << 16;
        else v[j >> 1] = *reinterpret_cast<const uint16_t*>(&e);
      }
    }
    const int64_t y = m / step;
    const int r = int(m - y * step), c = int(k >> 3) & 15;
    uint8_t* const to = out + ((b * chunks + y) * blocks + (k >> 7)) * (int64_t(kParts) * width * 256) + (c >> 3) * (width * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    if constexpr (kSplit) {
      uint4 w[3];
#pragma unroll
      for (int j = 0; j < 4; j++)
        split_pair(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), (&w[0].x)[j], (&w[1].x)[j], (&w[2].x)[j]);
#pragma unroll
      for (int q = 0; q < 3; q++) *reinterpret_cast<uint4*>(to + q * (width * 256)) = w[q];
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
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
  cudaLaunchAttribute attrs[2]{};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // begins while x is laid out
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = unsigned(shares);
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = shares > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, q4_many_kernel<kHalf, kPer>, p) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

}  // namespace

namespace emr {

emr_status q4_wait_error(int32_t* code, cudaStream_t st) { return take_wait_error(g_wait_error, code, st); }

// Rows of x of a block, their number as the instruction has it, and blocks along the rows.
static void columns_of(const Q4Product& a, int64_t* step, int64_t* width, int64_t* chunks) {
  const int64_t most = a.dtype == EMR_F32 ? 64 : 128;
  *chunks = (a.rows + most - 1) / most;
  *step = (a.rows + *chunks - 1) / *chunks;
  *width = (*step + 15) / 16 * 16;
}

size_t q4_many_room(const Q4Product& a) {
  int64_t step, width, chunks;
  columns_of(a, &step, &width, &chunks);
  return size_t(a.x_batch) * size_t(chunks) * size_t(q4_blocks(a.w->cols)) * size_t((a.dtype == EMR_F32 ? 3 : 1) * width * 256);
}

emr_status launch_q4_many(const Q4Product& a, void* ws, int dev, int sms, cudaStream_t st) {
  int64_t step, width, chunks;
  columns_of(a, &step, &width, &chunks);
  Params p{};
  p.w = a.w->data, p.tiles = int32_t(q4_tiles(a.w->rows)), p.blocks = int32_t(q4_blocks(a.w->cols)), p.row_blocks = (p.tiles + 7) / 8;
  p.w_batch = a.w->batch == 1 ? 0 : int64_t(p.tiles) * p.blocks * q4_unit(a.w->group);
  p.N = a.w->rows, p.M = a.rows;
  p.parts = a.dtype == EMR_F32 ? 3 : 1;
  p.bias = a.bias, p.act = a.act, p.out = a.out, p.out_dtype = a.out_dtype;
  const int64_t batch = a.x_batch > a.w->batch ? a.x_batch : a.w->batch, blocks = batch * p.row_blocks;
  if (chunks > 65535 || blocks > INT32_MAX / kMaxCluster) return EMR_ERR_RANGE;
  p.step = int(step), p.width = int(width);

  const int64_t total = int64_t(a.x_batch) * a.rows * p.blocks * 16, wanted = (total + 255) / 256;
  const unsigned grid = unsigned(wanted < 16 * sms ? wanted : 16 * sms);
  uint8_t* const out = static_cast<uint8_t*>(ws);
  // of both 16-bit types the bits are copied
  const emr_status laid = a.dtype == EMR_F32
                              ? launch_plain(q4_tiles_kernel<float>, dim3(grid), 256, st, static_cast<const float*>(a.x), a.rows, a.w->cols, p.blocks,
                                             a.batch_stride, a.row_stride, a.col_stride, a.whole, p.step, p.width, int(chunks), total, out)
                              : launch_plain(q4_tiles_kernel<__half>, dim3(grid), 256, st, static_cast<const __half*>(a.x), a.rows, a.w->cols, p.blocks,
                                             a.batch_stride, a.row_stride, a.col_stride, a.whole, p.step, p.width, int(chunks), total, out);
  if (laid != EMR_OK) return laid;
  p.x = out;
  p.x_batch = a.x_batch == 1 ? 0 : chunks * p.blocks * (int64_t(p.parts) * width * 256);

  int shares = 1;
  for (int s = 2; s <= kMaxCluster; s++)
    if (blocks * s * chunks <= sms && p.blocks / s >= 4) shares = s;
  const int room = kMostSmem - 1024 - kUnpack * kCodeStages * 32 * kRowPitch - kScale * 2 * kBatch, stage = p.parts * p.width * 256;
  p.stages = room / stage < kTileStages ? room / stage : kTileStages;
  const int per = kQ4Cols / a.w->group;
  if (a.dtype == EMR_F16)
    return per == 1 ? launch<true, 1>(p, blocks, shares, dev, st) : per == 2 ? launch<true, 2>(p, blocks, shares, dev, st) : launch<true, 4>(p, blocks, shares, dev, st);
  return per == 1 ? launch<false, 1>(p, blocks, shares, dev, st) : per == 2 ? launch<false, 2>(p, blocks, shares, dev, st) : launch<false, 4>(p, blocks, shares, dev, st);
}

}  // namespace emr
