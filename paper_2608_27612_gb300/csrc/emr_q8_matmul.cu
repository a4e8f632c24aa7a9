// Product of two block-scaled 8-bit matrices on the tensor cores:
//   out[b][m][n] = act(sum_k a[b][m][k] w[b][n][k] + bias[b][n]),
// optionally with act'(z) kept in 8 bits for the backward pass.
//
// With a = s_a q_a and w = s_w q_w and one scale for each row and block of 128
// columns, z = sum_kb s_a(m, kb) s_w(n, kb) sum_{k in kb} q_a q_w. The scales are
// powers of two in the format and granularity (a byte for each row, four blocks to a
// word) that the block-scaled matrix instruction reads from tensor memory, so they
// are applied inside it and no accumulator leaves tensor memory before the end of
// the contraction; the instruction's own blocks of 32 columns all take the byte of
// their block of 128.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>

#include <mutex>

#include "emr_act.h"
#include "emr_q8.h"
#include "emr_records.h"
#include "emr_tc.h"

namespace {

using namespace emr;

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
// Scale tile: 32 rows of 16 bytes, not swizzled, groups of 8 rows 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
  return uint64_t((addr & 0x3ffff) >> 4) | (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                           bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(uint32_t(accumulate))
      : "memory");
}
// ---- tiles ---------------------------------------------------------------------------

constexpr int kTileM = 128, kTileN = 128, kTileK = 128;
constexpr int kStages = 5;
constexpr int kOperandBytes = 128 * 128;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kScaleBytes = 1024;           // 512 for each operand
constexpr int kFinishWarps = 16;            // epilogue: four for each quarter of the rows, 32 columns each
constexpr int kStagingBytes = kFinishWarps * 32 * 64;  // 32 rows of 64 bytes a warp
constexpr int kThreads = 32 * (4 + kFinishWarps);      // copy warp, matrix warp, two that only wait, epilogue
constexpr int kTmemColumns = 512;
constexpr uint32_t kTmemScales = 256;       // behind the two accumulators of 128 columns
constexpr int kSmemBytes = 1024 + kStages * (kStageBytes + kScaleBytes) + kStagingBytes;

struct Params {
  int32_t M, N;
  int32_t m_tiles, n_tiles, tiles;  // tiles: over the batches of the output
  int32_t k_blocks, k_chunks;       // blocks of 128 columns, and scale chunks of four of them
  int32_t sum;                      // batches that one output sums over
  int32_t a_one, w_one;             // operand with batch 1
  const uint8_t *a_scales, *w_scales;
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype, store_bytes;   // store_bytes: widest store that every row of out is aligned to
  int32_t narrow;                   // at most 64 columns, no slopes: half of the epilogue's warps for each accumulator
  uint8_t *slope, *slope_scales;
  int32_t slope_whole;              // slope begins at a multiple of 32 bytes
};

struct Tile {
  int32_t b, m, n;
};
// Tiles in groups of 16 row tiles, so that the operand rows in use at a time stay in L2.
// 32-bit divisions: every warp makes them for every tile.
__device__ __forceinline__ Tile raster(uint32_t t, uint32_t m_tiles, uint32_t n_tiles, uint32_t tiles, uint32_t tall) {
  const uint32_t per = m_tiles * n_tiles, b = per == tiles ? 0 : t / per;
  t -= b * per;
  const uint32_t group = t / (tall * n_tiles), first = group * tall, rows = m_tiles - first < tall ? m_tiles - first : tall;
  t -= first * n_tiles;
  const uint32_t n = t / rows;
  return {int32_t(b), int32_t(first + t - n * rows), int32_t(n)};
}
__device__ __forceinline__ Tile tile_at(const Params& p, int t) { return raster(t, p.m_tiles, p.n_tiles, p.tiles, 16); }

// A warp's 32 staged rows of 64 bytes to global rows, sizeof(T) bytes a lane, neighbouring
// lanes neighbouring addresses. `bytes` are valid in each row, `rows` rows.
template <typename T>
__device__ __forceinline__ void store_rows(const uint8_t* staged, uint8_t* out, int64_t pitch, int rows, int bytes, int lane) {
  constexpr int kPer = 64 / int(sizeof(T));
  const int at = lane % kPer * int(sizeof(T));
#pragma unroll 4
  for (int r = lane / kPer; r < rows; r += 32 / kPer)
    if (at < bytes)
      *reinterpret_cast<T*>(out + r * pitch + at) =
          *reinterpret_cast<const T*>(staged + r * 64 + (((at >> 4) ^ ((r >> 1) & 3)) << 4) + (at & 15));
}
__device__ __forceinline__ void store_staged(const uint8_t* staged, uint8_t* out, int64_t pitch, int rows, int bytes, int width,
                                             int lane) {
  __syncwarp();
  if (width == 16) store_rows<uint4>(staged, out, pitch, rows, bytes, lane);
  else if (width == 8) store_rows<uint2>(staged, out, pitch, rows, bytes, lane);
  else if (width == 4) store_rows<uint32_t>(staged, out, pitch, rows, bytes, lane);
  else store_rows<uint16_t>(staged, out, pitch, rows, bytes, lane);
  __syncwarp();
}
__device__ __forceinline__ void stage16(uint8_t* staged, int row, int unit, uint4 v) {
  *reinterpret_cast<uint4*>(staged + row * 64 + ((unit ^ ((row >> 1) & 3)) << 4)) = v;
}
__device__ __forceinline__ uint32_t pack_half(int dtype, float a, float b) {
  if (dtype == EMR_BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// What the epilogue's warps share; read in pieces of 16 bytes.
struct alignas(16) Finish {
  float tops[2][128][4];  // largest slope of a row's 32 columns, two turns
  float bias[kFinishWarps][32];
};
static_assert(offsetof(Finish, bias) % 16 == 0, "rows of bias begin at multiples of 16 bytes");
// 32 bytes to an address that is a multiple of 16; `whole`: of 32, which one store of them asks for.
// Predicated: a branch made the pair kernel spill.
__device__ __forceinline__ void store32(uint8_t* to, const uint32_t (&w)[8], int32_t whole) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %9, 0;\n\t"
      "@p st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n\t"
      "@!p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\t"
      "@!p st.global.v4.b32 [%0 + 16], {%5, %6, %7, %8};\n\t}" ::"l"(to),
      "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(whole)
      : "memory");
}

// A warp's 32 rows and 32 columns (c-th of four) of one 128-column accumulator block at tensor
// memory address addr: bias, activation, output and, with kSlope, slope. read() is called
// when the accumulators have been read. Sixteen warps share a block because a warp by itself
// issues an instruction only every four or five clocks, and in chunks of 32 columns because the
// code of more, unrolled, does not stay in the instruction cache.
template <bool kSlope, typename Read>
__device__ __forceinline__ void finish_chunk(const Params& p, const Tile& t, uint32_t addr, int c, float bias, uint8_t* staged,
                                             Finish& share, uint32_t turn, int row0, int warp, int lane, Read read) {
  const int n0 = t.n * kTileN + c * 32;
  const int rows = p.M - row0 < 32 ? p.M - row0 : 32;
  const int cols = p.N - n0 < 32 ? p.N - n0 : 32;  // may be below 1
  const int64_t first = (int64_t(t.b) * p.M + row0) * p.N + n0;
  float z[32], d[32];
  tmem_load32(addr + c * 32, z);
  fence_before();
  read();
  if (p.bias) {
    float* const own = share.bias[warp];
    own[lane] = bias;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float4 b = reinterpret_cast<const float4*>(own)[i];
      z[4 * i] += b.x, z[4 * i + 1] += b.y, z[4 * i + 2] += b.z, z[4 * i + 3] += b.w;
    }
    __syncwarp();
  }
  if (rows < 32 || cols < 32) {  // scales past the matrix are any bytes: what they gave stays out of the activation
#pragma unroll
    for (int i = 0; i < 32; i++) z[i] = lane < rows && i < cols ? z[i] : 0.f;
  }
  activate<32, kSlope>(p.act, z, d);
  if (p.out_dtype == EMR_F32) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int j = h * 16 + i * 4;
        stage16(staged, lane, i, make_uint4(__float_as_uint(z[j]), __float_as_uint(z[j + 1]), __float_as_uint(z[j + 2]), __float_as_uint(z[j + 3])));
      }
      const int left = (cols - h * 16) * 4;
      store_staged(staged, static_cast<uint8_t*>(p.out) + (first + h * 16) * 4, int64_t(p.N) * 4, rows,
                   left < 64 ? left : 64, p.store_bytes, lane);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      stage16(staged, lane, i,
              make_uint4(pack_half(p.out_dtype, z[8 * i], z[8 * i + 1]), pack_half(p.out_dtype, z[8 * i + 2], z[8 * i + 3]),
                         pack_half(p.out_dtype, z[8 * i + 4], z[8 * i + 5]), pack_half(p.out_dtype, z[8 * i + 6], z[8 * i + 7])));
    store_staged(staged, static_cast<uint8_t*>(p.out) + first * 2, int64_t(p.N) * 2, rows, cols * 2, p.store_bytes, lane);
  }
  if constexpr (kSlope) {
    if (cols < 32) {
#pragma unroll
      for (int i = 0; i < 32; i++) d[i] = i < cols ? d[i] : 0.f;
    }
    float top = 0.f;  // slopes are finite or NaN, which the maxima pass over
#pragma unroll
    for (int i = 0; i < 32; i++) top = fmaxf(top, fabsf(d[i]));
    const int quadrant = warp & 3;
    float(&tops)[4] = share.tops[turn & 1][quadrant * 32 + lane];
    tops[c] = top;
    asm volatile("bar.sync %0, 128;" ::"r"(1 + quadrant) : "memory");  // the row's four warps
    const float4 all = *reinterpret_cast<const float4*>(tops);
    const uint32_t byte = q8_scale_byte(__float_as_uint(fmaxf(fmaxf(all.x, all.y), fmaxf(all.z, all.w))));
    const float inv = q8_inverse(byte);
    if (lane < rows) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; i++) w[i] = q8_pack4(d[4 * i], d[4 * i + 1], d[4 * i + 2], d[4 * i + 3], inv);
      const int row = row0 + lane;
      store32(p.slope + (int64_t(t.b) * p.M + row) * q8_row_bytes(p.N) + n0, w, p.slope_whole);
      if (c == 0) p.slope_scales[t.b * q8_scale_batch(p.M, p.N) + q8_scale_at(q8_scale_chunks(p.N), row, t.n)] = uint8_t(byte);
    }
  }
}

constexpr int kFinishBarrier = 5;  // of all epilogue warps; 1 to 4 are the quarters
__device__ __forceinline__ void finish_sync() { asm volatile("bar.sync %0, %1;" ::"n"(kFinishBarrier), "n"(32 * kFinishWarps) : "memory"); }
// Whether the accumulators of a tile are there; with kSlope with one answer for the warps that then
// meet at barriers while finishing the tile: `count` threads at barrier `id`.
template <bool kSlope>
__device__ __forceinline__ bool finish_wait(uint32_t bar, uint32_t parity, volatile int* stop, int code, int id, int count) {
  const bool ok = warp_wait(bar, parity, stop, code);
  if (!kSlope) return ok;
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(uint32_t(ok)), "r"(id), "r"(count)
      : "memory");
  return all != 0;
}

// Persistent: a block takes tiles blockIdx.x, + gridDim.x, ... Warp 0 copies operand and
// scale tiles into a ring of stages, warp 1 issues the matrix instructions, warps 4..19
// finish a tile while the next one accumulates in the other half of tensor memory.
template <bool kSlope>
__global__ void __launch_bounds__(kThreads, 1) q8_matmul_kernel(const __grid_constant__ CUtensorMap a_map,
                                                                const __grid_constant__ CUtensorMap w_map,
                                                                const __grid_constant__ Params p) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 4];
  __shared__ Finish share;
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  uint8_t* const sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* const scales_sm = sm + kStages * kStageBytes;
  uint8_t* const staging = scales_sm + kStages * kScaleBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full = smem_at(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
  volatile int* const stop = &gave_up;

  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < kStages; i++) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    for (int i = 0; i < 2; i++) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, p.narrow ? kFinishWarps / 2 : kFinishWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_base)), "n"(kTmemColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_base;
  grid_wait();
  grid_go();
  const int steps = p.sum * p.k_blocks;

  if (warp == 0) {
    Ring<kStages> ring;
    for (int t = blockIdx.x; t < p.tiles && !*stop; t += gridDim.x) {
      const Tile tile = tile_at(p, t);
      const int m = tile.m * kTileM, n = tile.n * kTileN;
      bool ok = true;
      for (int sb = 0; sb < p.sum && ok; sb++) {
        const int b = tile.b + sb, ab = p.a_one ? 0 : b, wb = p.w_one ? 0 : b;
        const uint8_t* a_scales = p.a_scales + (int64_t(ab) * p.m_tiles + tile.m) * p.k_chunks * 512;
        const uint8_t* w_scales = p.w_scales + (int64_t(wb) * p.n_tiles + tile.n) * p.k_chunks * 512;
        for (int kb = 0; kb < p.k_blocks; kb++, ring.next()) {
          // a new ring is empty: the wait for the round before the first returns at once
          if (!(ok = warp_wait(empty + 8 * ring.stage, ring.round ^ 1, stop, 1))) break;
          const uint32_t bar = full + 8 * ring.stage, dst = smem_at(sm) + ring.stage * kStageBytes;
          const bool scales = (kb & 3) == 0;
          if (elect_one()) {
            bar_expect(bar, kStageBytes + (scales ? kScaleBytes : 0));
            tma_load(dst, &a_map, kb * kTileK, m, ab, bar);
            tma_load(dst + kOperandBytes, &w_map, kb * kTileK, n, wb, bar);
            if (scales) {
              const uint32_t at = smem_at(scales_sm) + ring.stage * kScaleBytes;
              bulk_load(at, a_scales, 512, bar);
              bulk_load(at + 512, w_scales, 512, bar);
            }
          }
          __syncwarp();
          if (scales) a_scales += 512, w_scales += 512;
        }
      }
    }
    if (*stop) settle();
  } else if (warp == 1) {
    const uint32_t idesc = (1u << 23) | (uint32_t(kTileN >> 3) << 17) | (uint32_t(kTileM >> 4) << 24);
    Ring<kStages> ring;
    uint32_t n_tile = 0, chunk = 0;
    for (int t = blockIdx.x; t < p.tiles && !*stop; t += gridDim.x, n_tile++) {
      const uint32_t acc = n_tile & 1;
      if (n_tile >= 2 && !warp_wait(acc_empty + 8 * acc, ((n_tile >> 1) - 1) & 1, stop, 2)) break;
      fence_after();
      uint32_t sf = 0;
      for (int k = 0, kb = 0; k < steps; k++, ring.next()) {
        const int s = ring.stage;
        if (!warp_wait(full + 8 * s, ring.round, stop, 3)) break;
        fence_after();
        if ((kb & 3) == 0) {
          sf = tmem + kTmemScales + 8 * (chunk++ & 1);
          const uint32_t at = smem_at(scales_sm) + s * kScaleBytes;
          if (elect_one()) {
            copy_scales(sf, scale_desc(at));
            copy_scales(sf + 4, scale_desc(at + 512));
          }
          __syncwarp();
        }
        const uint32_t at = smem_at(sm) + s * kStageBytes;
        const uint64_t a = operand_desc(at), w = operand_desc(at + kOperandBytes);
        const uint32_t id = idesc | (uint32_t(kb & 3) << 4) | (uint32_t(kb & 3) << 29);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < 4; j++)  // 32 columns each: 32 bytes further in the tile
            mma_scaled(tmem + acc * kTileN, a + 2 * j, w + 2 * j, id, sf, sf + 4, k > 0 || j > 0);
          mma_commit(empty + 8 * s);
        }
        __syncwarp();
        if (++kb == p.k_blocks) kb = 0;
      }
      if (elect_one()) mma_commit(acc_full + 8 * acc);
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int quadrant = warp & 3;  // tensor memory lanes that this warp may read
    // with at most 64 columns the warps of the other two chunks take every other tile: 112 networks
    // of 13496 x 45 x 86 195 -> 134 us
    const int own = warp - 4, c = p.narrow ? own >> 2 & 1 : own >> 2, group = own >> 3;
    uint8_t* const staged = staging + own * 32 * 64;
    uint32_t n_tile = 0;
    for (int t = blockIdx.x; t < p.tiles; t += gridDim.x, n_tile++) {
      const uint32_t acc = n_tile & 1;
      if (!kSlope && p.narrow && int(acc) != group) continue;
      const Tile tile = tile_at(p, t);
      const int row0 = tile.m * kTileM + quadrant * 32, n = tile.n * kTileN + c * 32 + lane;
      const float bias = p.bias && n < p.N ? __ldg(p.bias + int64_t(tile.b) * p.N + n) : 0.f;
      if (!finish_wait<kSlope>(acc_full + 8 * acc, (n_tile >> 1) & 1, stop, 4, 1 + quadrant, 128)) break;
      fence_after();
      if (row0 >= p.M || (!kSlope && n - lane >= p.N)) {  // nothing of this warp's part is in the matrix
        if (lane == 0) bar_arrive(acc_empty + 8 * acc);
        __syncwarp();
        continue;
      }
      const uint32_t addr = tmem + acc * kTileN + (uint32_t(quadrant * 32) << 16);
      finish_chunk<kSlope>(p, tile, addr, c, bias, staged, share, n_tile, row0, own, lane, [&] {
        if (lane == 0) bar_arrive(acc_empty + 8 * acc);
      });
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColumns) : "memory");
  }
}

// ---- pairs of SMs --------------------------------------------------------------------
// For large products the 128 x 128 tile is bound by what L2 delivers: 32 KB an SM for each
// 256 clocks of matrix work. Two SMs of a cluster on one 256 x 256 tile take 32 KB each for
// 512 clocks: either block stages 128 rows of each operand, and the matrix instructions,
// issued by the first block, read both blocks' shared memory and write 128 x 256
// accumulators in each. Two such accumulators fill tensor memory, so the scales of one tile
// live in the last 24 columns of the other tile's accumulators, which the epilogue reads
// first.

constexpr int kPairStages = 5;
constexpr int kPairScaleBytes = 1536;  // 512 of a, 1024 of w
constexpr int kPairSmemBytes = 1024 + kPairStages * (kStageBytes + kPairScaleBytes) + kStagingBytes;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's window, of the first block's copy of a shared address.
__device__ __forceinline__ uint32_t at_first(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_load_scales(uint32_t dst, const CUtensorMap* map, int tile, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(0), "r"(tile), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(uint32_t(accumulate))
      : "memory");
}
// Arrives at the barrier's address in both blocks when the work issued so far is done.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"(uint16_t(3))
               : "memory");
}

// Tile t of the pairs' raster: b, and row and column of 256 (groups of 8 row tiles).
__device__ __forceinline__ Tile pair_tile_at(const Params& p, int t) {
  return raster(t, (p.m_tiles + 1) / 2, (p.n_tiles + 1) / 2, p.tiles, 8);
}

// The same on pairs of SMs: 256 x 256 tiles, half the operand bytes for each output. Loads
// bound a single SM's tiles (540 clocks a step of 128 columns, 61 bytes a clock from L2, where
// the matrix instructions take 256); of a pair's time at 8192^3 loads alone would take 209
// us and the instructions 271. 8192^3 305 us (3.6 PFLOP/s), with slopes 321; 94464 x 1364 x 1364
// 140, with sin 179.
template <bool kSlope>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    q8_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap w_map,
                   const __grid_constant__ CUtensorMap a_scale_map, const __grid_constant__ CUtensorMap w_scale_map,
                   const __grid_constant__ Params p) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kPairStages + 6];
  __shared__ Finish share;
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  // the dynamic part starts at the same address in both blocks
  uint8_t* const sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* const scales_sm = sm + kPairStages * kStageBytes;
  uint8_t* const staging = scales_sm + kPairStages * kPairScaleBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t full = smem_at(bars), empty = full + 8 * kPairStages, acc_full = empty + 8 * kPairStages,
                 acc_empty = acc_full + 16, tail = acc_empty + 16;
  volatile int* const stop = &gave_up;

  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < kPairStages; i++) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    for (int i = 0; i < 2; i++) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, 2 * kFinishWarps), bar_init(tail + 8 * i, 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_base)), "n"(kTmemColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  cluster_sync();
  fence_after();
  const uint32_t tmem = tmem_base;
  grid_wait();
  grid_go();
  const int steps = p.sum * p.k_blocks;
  const int stride = gridDim.x / 2, start = blockIdx.x / 2;
  if (warp == 0) {
    Ring<kPairStages> ring;
    for (int t = start; t < p.tiles && !*stop; t += stride) {
      const Tile tile = pair_tile_at(p, t);
      const int m = tile.m * 2 + int(rank), n = tile.n * 2 + int(rank);
      const int m_scale = m < p.m_tiles ? m : p.m_tiles - 1;
      const int next = tile.n * 2 + 1 < p.n_tiles ? p.k_chunks : 0;  // scale tiles on to w's second 128 rows
      bool ok = true;
      for (int sb = 0; sb < p.sum && ok; sb++) {
        const int b = tile.b + sb, ab = p.a_one ? 0 : b, wb = p.w_one ? 0 : b;
        int a_scales = (ab * p.m_tiles + m_scale) * p.k_chunks, w_scales = (wb * p.n_tiles + tile.n * 2) * p.k_chunks;
        for (int kb = 0; kb < p.k_blocks; kb++, ring.next()) {
          if (!(ok = warp_wait(empty + 8 * ring.stage, ring.round ^ 1, stop, 5))) break;
          const uint32_t dst = smem_at(sm) + ring.stage * kStageBytes, bar = at_first(full + 8 * ring.stage);
          const bool scales = (kb & 3) == 0;
          if (elect_one()) {
            if (rank == 0) bar_expect(full + 8 * ring.stage, 2 * (kStageBytes + (scales ? kPairScaleBytes : 0)));
            pair_load(dst, &a_map, kb * kTileK, m * kTileM, ab, bar);
            pair_load(dst + kOperandBytes, &w_map, kb * kTileK, n * kTileN, wb, bar);
            if (scales) {
              const uint32_t at = smem_at(scales_sm) + ring.stage * kPairScaleBytes;
              pair_load_scales(at, &a_scale_map, a_scales, bar);
              pair_load_scales(at + 512, &w_scale_map, w_scales, bar);
              pair_load_scales(at + 1024, &w_scale_map, w_scales + next, bar);
            }
          }
          __syncwarp();
          if (scales) a_scales++, w_scales++;
        }
      }
    }
    if (*stop) settle();
  } else if (warp == 1 && rank == 0) {
    const uint32_t idesc = (1u << 23) | (uint32_t(256 >> 3) << 17) | (uint32_t(256 >> 4) << 24);
    Ring<kPairStages> ring;
    uint32_t n_tile = 0, chunk = 0;
    for (int t = start; t < p.tiles && !*stop; t += stride, n_tile++) {
      const uint32_t acc = n_tile & 1, other = acc ^ 1;
      if (n_tile >= 2 && !warp_wait(acc_empty + 8 * acc, ((n_tile >> 1) - 1) & 1, stop, 6)) break;
      if (n_tile >= 1 && !warp_wait(tail + 8 * other, ((n_tile - 1) >> 1) & 1, stop, 7)) break;
      fence_after();
      uint32_t sfa = 0, sfw = 0;
      for (int k = 0, kb = 0; k < steps; k++, ring.next()) {
        const int s = ring.stage;
        if (!warp_wait(full + 8 * s, ring.round, stop, 8)) break;
        fence_after();
        if ((kb & 3) == 0) {
          const uint32_t turn = chunk++ & 1, at = smem_at(scales_sm) + s * kPairScaleBytes;
          sfw = tmem + other * 256 + 232 + 8 * turn;
          sfa = tmem + other * 256 + 248 + 4 * turn;
          if (elect_one()) {
            pair_copy_scales(sfa, scale_desc(at));
            pair_copy_scales(sfw, scale_desc(at + 512));
            pair_copy_scales(sfw + 4, scale_desc(at + 1024));
          }
          __syncwarp();
        }
        const uint32_t at = smem_at(sm) + s * kStageBytes;
        const uint64_t a = operand_desc(at), w = operand_desc(at + kOperandBytes);
        const uint32_t id = idesc | (uint32_t(kb & 3) << 4) | (uint32_t(kb & 3) << 29);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < 4; j++) pair_mma(tmem + acc * 256, a + 2 * j, w + 2 * j, id, sfa, sfw, k > 0 || j > 0);
          pair_commit(empty + 8 * s);
        }
        __syncwarp();
        if (++kb == p.k_blocks) kb = 0;
      }
      if (elect_one()) pair_commit(acc_full + 8 * acc);
      __syncwarp();
    }
  } else if (warp >= 4) {
    const int quadrant = warp & 3, own = warp - 4, c = own >> 2;
    uint8_t* const staged = staging + own * 32 * 64;
    uint32_t n_tile = 0, turn = 0;
    for (int t = start; t < p.tiles; t += stride, n_tile++) {
      const uint32_t acc = n_tile & 1;
      const Tile pair = pair_tile_at(p, t);
      const int row0 = (pair.m * 2 + int(rank)) * kTileM + quadrant * 32;
      const uint32_t addr = tmem + acc * 256 + (uint32_t(quadrant * 32) << 16);
      const uint32_t done = at_first(acc_empty + 8 * acc), last = at_first(tail + 8 * acc);
#pragma unroll 1
      for (int half = 1; half >= 0; half--, turn++) {  // the scales' columns first
        const Tile tile{pair.b, pair.m * 2 + int(rank), pair.n * 2 + half};
        const int n = tile.n * kTileN + c * 32 + lane;
        const float bias = p.bias && n < p.N ? __ldg(p.bias + int64_t(tile.b) * p.N + n) : 0.f;
        if (half) {
          if (!finish_wait<kSlope>(acc_full + 8 * acc, (n_tile >> 1) & 1, stop, 9, kFinishBarrier, 32 * kFinishWarps)) goto out;
          fence_after();
        }
        // The columns that the next tile's scales are waiting for are read before all others; without
        // slopes the epilogue is short and the barrier costs more than it saves (with slopes
        // 8192^3 334 us without, 321 with).
        const bool scales = half && c == 3;
        if (kSlope && half && !scales) finish_sync();
        auto read = [&] {
          if (lane == 0) {
            if (scales) bar_arrive_cluster(last);
            if (!half) bar_arrive_cluster(done);
          }
          __syncwarp();
          if (kSlope && scales) finish_sync();
        };
        if (row0 >= p.M || tile.n >= p.n_tiles || (!kSlope && n - lane >= p.N)) {  // nothing of this warp's part is in the matrix
          read();
          __syncwarp();
          continue;
        }
        finish_chunk<kSlope>(p, tile, addr + half * 128, c, bias, staged, share, turn, row0, own, lane, read);
      }
    }
  out:;
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  cluster_sync();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColumns) : "memory");
  }
}

// ---- few rows, or few tiles ---------------------------------------------------------
// With few rows of a the weights' bytes bound the product, and a tile of 128 outputs for
// each SM leaves most of them without work. Here the operands change places: 128 rows of
// w are the instruction's rows and the rows of a, 16 to 128 of them, its columns, so a
// block streams little but weights; two blocks share an SM, and the blocks of a cluster
// share the contraction of one tile and add their accumulators, through each other's
// shared memory, in the order of their ranks. A lane of the epilogue has one output of
// each row, so its stores are neighbours. The same kernel serves larger a with few tiles
// and a long contraction (the gradient of an input that many networks share). 8 x 8192 x
// 8192: 9.8 us with the weights in L2, 20 from memory (3.3 TB/s), where tiles of 128 rows took
// 21 and 31; 250 x 256 summed over 64 networks of 340: 57 -> 11 us
// (13 with clusters of 8).

constexpr int kThinStages = 6;     // at most; q.stages of them are used
constexpr int kThinThreads = 320;  // copy warp, matrix warp, eight epilogue warps
constexpr int kThinColumns = 256;  // of tensor memory: half of it

struct ThinParams {
  Params p;
  int32_t wide;   // rows of a in a tile: 16, 32, 64 or 128
  int32_t split;  // blocks of a cluster
  int32_t stages;
};
__host__ __device__ inline int thin_stage_bytes(int wide) { return kOperandBytes + wide * 128 + kScaleBytes; }

__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r[i]);
}
// The address, in the cluster's window, of block `rank`'s copy of a shared address.
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

__global__ void __launch_bounds__(kThinThreads, 2) q8_thin_kernel(const __grid_constant__ CUtensorMap a_map,
                                                                  const __grid_constant__ CUtensorMap w_map,
                                                                  const __grid_constant__ ThinParams q) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kThinStages + 4];
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  const Params& p = q.p;
  uint8_t* const sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const int wide_bytes = q.wide * 128;
  uint8_t* const rows_sm = sm + q.stages * kOperandBytes;
  uint8_t* const scales_sm = rows_sm + q.stages * wide_bytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full = smem_at(bars), empty = full + 8 * kThinStages, acc_full = empty + 8 * kThinStages, acc_empty = acc_full + 16;
  volatile int* const stop = &gave_up;
  const int rank = q.split > 1 ? int(cluster_rank()) : 0;
  const int steps = p.sum * p.k_blocks;
  const int first = int(int64_t(steps) * rank / q.split), last = int(int64_t(steps) * (rank + 1) / q.split);
  const int first_sb = first / p.k_blocks, first_kb = first - first_sb * p.k_blocks;
  const int accs = q.wide <= 64 ? 2 : 1;  // accumulators at columns 0 and 64, scales from 128 on (wide 128: from 128)

  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < kThinStages; i++) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    for (int i = 0; i < 2; i++) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_base)), "n"(kThinColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_base;
  grid_wait();
  grid_go();
  const int stride = int(gridDim.x) / q.split, start = int(blockIdx.x) / q.split;

  if (warp == 0) {
    int stage = 0;
    uint32_t round = 0;
    const auto next = [&] {
      if (++stage == q.stages) stage = 0, round ^= 1;
    };
    for (int t = start; t < p.tiles && !*stop; t += stride) {
      const Tile tile = tile_at(p, t);
      int kb = first_kb, sb = first_sb;
      for (int i = first; i < last; i++, next()) {
        if (!warp_wait(empty + 8 * stage, round ^ 1, stop, 10)) break;
        const int b = tile.b + sb, ab = p.a_one ? 0 : b, wb = p.w_one ? 0 : b;
        if (elect_one()) {
          const uint32_t bar = full + 8 * stage;
          const bool scales = i == first || (kb & 3) == 0;
          bar_expect(bar, kOperandBytes + wide_bytes + (scales ? kScaleBytes : 0));
          tma_load(smem_at(sm) + stage * kOperandBytes, &w_map, kb * kTileK, tile.n * kTileN, wb, bar);
          tma_load(smem_at(rows_sm) + stage * wide_bytes, &a_map, kb * kTileK, tile.m * kTileM, ab, bar);
          if (scales) {
            const uint32_t at = smem_at(scales_sm) + stage * kScaleBytes;
            bulk_load(at, p.w_scales + ((int64_t(wb) * p.n_tiles + tile.n) * p.k_chunks + (kb >> 2)) * 512, 512, bar);
            bulk_load(at + 512, p.a_scales + ((int64_t(ab) * p.m_tiles + tile.m) * p.k_chunks + (kb >> 2)) * 512, 512, bar);
          }
        }
        if (++kb == p.k_blocks) kb = 0, sb++;
        __syncwarp();
      }
    }
    if (*stop) settle();
  } else if (warp == 1) {
    const uint32_t idesc = (1u << 23) | (uint32_t(q.wide >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    int stage = 0;
    uint32_t round = 0;
    const auto next = [&] {
      if (++stage == q.stages) stage = 0, round ^= 1;
    };
    uint32_t n_tile = 0, chunk = 0;
    for (int t = start; t < p.tiles && !*stop; t += stride, n_tile++) {
      const uint32_t acc = accs == 2 ? n_tile & 1 : 0, use = accs == 2 ? n_tile >> 1 : n_tile;
      if (use >= 1 && !warp_wait(acc_empty + 8 * acc, (use - 1) & 1, stop, 11)) break;
      fence_after();
      uint32_t sf = 0;
      int kb = first_kb;
      for (int i = first; i < last; i++, next()) {
        const int s = stage;
        if (!warp_wait(full + 8 * s, round, stop, 12)) break;
        fence_after();
        if (i == first || (kb & 3) == 0) {
          sf = tmem + 128 + 8 * (chunk++ & 1);
          const uint32_t at = smem_at(scales_sm) + s * kScaleBytes;
          if (elect_one()) {
            copy_scales(sf, scale_desc(at));
            copy_scales(sf + 4, scale_desc(at + 512));
          }
          __syncwarp();
        }
        const uint64_t w = operand_desc(smem_at(sm) + s * kOperandBytes), a = operand_desc(smem_at(rows_sm) + s * wide_bytes);
        const uint32_t id = idesc | (uint32_t(kb & 3) << 4) | (uint32_t(kb & 3) << 29);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < 4; j++) mma_scaled(tmem + acc * 64, w + 2 * j, a + 2 * j, id, sf, sf + 4, i > first || j > 0);
          mma_commit(empty + 8 * s);
        }
        __syncwarp();
        if (++kb == p.k_blocks) kb = 0;
      }
      if (elect_one()) mma_commit(acc_full + 8 * acc);
      __syncwarp();
    }
  } else {
    const int row = (warp & 3) * 32 + lane;  // of the tile's 128 outputs; the second four warps take every other 16 rows of a
    const int half = (warp - 2) >> 2;
    uint32_t n_tile = 0;
    for (int t = start; t < p.tiles; t += stride, n_tile++) {
      const Tile tile = tile_at(p, t);
      const int b = tile.b, n = tile.n * kTileN + row, m0 = tile.m * kTileM;
      const uint32_t acc = accs == 2 ? n_tile & 1 : 0, use = accs == 2 ? n_tile >> 1 : n_tile;
      const float bias = q.split == 1 && p.bias && n < p.N ? __ldg(p.bias + int64_t(b) * p.N + n) : 0.f;
      if (!warp_wait(acc_full + 8 * acc, use & 1, stop, 13)) break;
      fence_after();
      const uint32_t addr = tmem + acc * 64 + (uint32_t((warp & 3) * 32) << 16);
#pragma unroll 1
      for (int c = half * 16; c < q.wide; c += 32) {
        float z[16], d[16];
        tmem_load16(addr + c, z);
        if (q.split > 1) {  // this block's share, [row of a][output]; the stages are done with
          float* const share = reinterpret_cast<float*>(sm);
#pragma unroll
          for (int i = 0; i < 16; i++) share[(c + i) * 128 + row] = z[i];
          continue;
        }
        if (n < p.N) {
#pragma unroll
          for (int i = 0; i < 16; i++) z[i] = m0 + c + i < p.M ? z[i] + bias : 0.f;
          activate<16, false>(p.act, z, d);
#pragma unroll
          for (int i = 0; i < 16; i++)
            if (m0 + c + i < p.M) store_scalar(p.out, p.out_dtype, (int64_t(b) * p.M + m0 + c + i) * p.N + n, z[i]);
        }
      }
      fence_before();
      if (lane == 0) bar_arrive(acc_empty + 8 * acc);
      __syncwarp();
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (q.split > 1) {  // one tile a cluster
    cluster_sync();
    const Tile tile = tile_at(p, start);
    const int b = tile.b, n0 = tile.n * kTileN, m0 = tile.m * kTileM, have = p.M - m0 < q.wide ? p.M - m0 : q.wide;
    const bool fine = !*stop;
    // four neighbouring outputs of a row at a time, rows shared out over the blocks
    for (int i = threadIdx.x; i < 32 * ((have - rank + q.split - 1) / q.split); i += kThinThreads) {
      const int m = (i >> 5) * q.split + rank, r = (i & 31) * 4;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < q.split; s++) {
        const float4 v = cluster_load4(at_rank(smem_at(sm) + (m * 128 + r) * 4, s));
        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
      }
      float z[4] = {sum.x, sum.y, sum.z, sum.w}, d[4];
#pragma unroll
      for (int j = 0; j < 4; j++) z[j] = n0 + r + j < p.N ? z[j] + (p.bias ? __ldg(p.bias + int64_t(b) * p.N + n0 + r + j) : 0.f) : 0.f;
      activate<4, false>(p.act, z, d);
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (fine && n0 + r + j < p.N) store_scalar(p.out, p.out_dtype, (int64_t(b) * p.M + m0 + m) * p.N + n0 + r + j, z[j]);
    }
    cluster_sync();  // no block ends while another reads its share
  }
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kThinColumns) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static std::once_flag once;
  static EncodeTiled fn = nullptr;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) == cudaSuccess &&
        found == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiled>(p);
  });
  return fn;
}

// Boxes of `rows` rows x 128 columns of a q8 matrix; rows past it read as zeros.
bool operand_map(const emr_q8* q, CUtensorMap* map, int rows = 128) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t row_bytes = cuuint64_t(q8_row_bytes(q->cols));
  const cuuint64_t dims[3] = {row_bytes, cuuint64_t(q->rows), cuuint64_t(q->batch)};
  const cuuint64_t strides[2] = {row_bytes, row_bytes * cuuint64_t(q->rows)};
  const cuuint32_t box[3] = {128, cuuint32_t(rows), 1}, ones[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, q->values, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The 512-byte scale tiles of a q8 matrix, one a row.
bool scale_map(const emr_q8* q, CUtensorMap* map) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t tiles = cuuint64_t(q->batch) * q8_scale_batch(q->rows, q->cols) / 512;
  const cuuint64_t dims[2] = {128, tiles}, strides[1] = {512};
  const cuuint32_t box[2] = {128, 1}, ones[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, q->scales, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kSlope>
emr_status launch_pairs(const emr_q8* a, const emr_q8* w, const CUtensorMap& a_map, const CUtensorMap& w_map, Params p, int dev, int sms,
                        cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap a_scales, w_scales;
  if (!scale_map(a, &a_scales) || !scale_map(w, &w_scales)) return EMR_ERR_CUDA;
  if (!allow_smem(q8_pair_kernel<kSlope>, kPairSmemBytes, dev, done)) return EMR_ERR_CUDA;
  p.tiles = p.tiles / (p.m_tiles * p.n_tiles) * ((p.m_tiles + 1) / 2) * ((p.n_tiles + 1) / 2);
  const int64_t pairs = sms / 2;
  return launch_after(q8_pair_kernel<kSlope>, dim3(unsigned(2 * (p.tiles < pairs ? p.tiles : pairs))), kThreads, kPairSmemBytes, st, a_map,
                      w_map, a_scales, w_scales, p);
}

template <bool kSlope>
emr_status launch(const CUtensorMap& a, const CUtensorMap& w, const Params& p, int dev, int sms, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(q8_matmul_kernel<kSlope>, kSmemBytes, dev, done)) return EMR_ERR_CUDA;
  return launch_after(q8_matmul_kernel<kSlope>, dim3(unsigned(p.tiles < sms ? p.tiles : sms)), kThreads, kSmemBytes, st, a, w, p);
}

// Clusters of 16 blocks of the thin kernel that run at once (0: none), asked once for each device
// and kind of block.
int clusters_of_16(int dev, bool small, size_t smem) {
  static std::atomic<int> known[64][2];  // 1 + the answer
  if (dev >= 64) return 0;
  std::atomic<int>& slot = known[dev][small];
  int n = slot.load(std::memory_order_relaxed);
  if (n == 0) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(kThinThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 16, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int fit = 0;
    if (cudaFuncSetAttribute(q8_thin_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&fit, q8_thin_kernel, &cfg) != cudaSuccess)
      fit = 0, cudaGetLastError();  // the question's error is not the caller's
    n = 1 + fit;
    slot.store(n, std::memory_order_relaxed);
  }
  return n - 1;
}

emr_status launch_thin(const emr_q8* a, const emr_q8* w, const Params& p, int dev, int sms, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  ThinParams q{};
  q.p = p;
  q.wide = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
  // As many blocks to a tile as find room, with two blocks of columns for each; 16 of them, which not
  // every device takes, where that many clusters run at once.
  q.split = 1;
  const int64_t room = q.wide <= 64 ? 2 * sms : sms;  // 100 KB a block up to 64 rows
  const auto more = [&] { return int64_t(p.tiles) * q.split * 2 <= room && int64_t(p.sum) * p.k_blocks >= 4 * q.split; };
  while (q.split < 8 && more()) q.split *= 2;
  CUtensorMap a_map, w_map;
  if (!operand_map(a, &a_map, q.wide) || !operand_map(w, &w_map)) return EMR_ERR_CUDA;
  q.stages = q.wide <= 64 ? 4 : 6;
  const int smem = 1024 + q.stages * thin_stage_bytes(q.wide);  // the shares, wide rows of 512 bytes, fit in w's stages
  if (!allow_smem(q8_thin_kernel, 1024 + kThinStages * thin_stage_bytes(128), dev, done)) return EMR_ERR_CUDA;
  if (q.split == 8 && more() && p.tiles <= clusters_of_16(dev, q.wide <= 64, size_t(smem))) q.split = 16;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(q.split > 1 ? p.tiles * q.split : p.tiles < room ? p.tiles : room));
  cfg.blockDim = dim3(kThinThreads);
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(q.split);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = q.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, q8_thin_kernel, a_map, w_map, q) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

// At most 64 rows, or so few tiles of a long contraction that most SMs would have none. From 65
// rows on the exchanged operands save no bytes: 100 x 8192 x 300 8.1 us by this kernel and 4.6 by
// tiles, 26 networks of 98 x 5965 x 74 58 and 29; of 64 x 5965 x 74 23 and 29.
bool use_thin(const Params& p, int sms) {
  if (p.M <= 64) return true;
  return int64_t(p.tiles) * 2 <= sms && int64_t(p.sum) * p.k_blocks >= 16;
}

// Pairs of SMs where their rounds of 256 x 256 tiles take less time than one SM's rounds of
// 128 x 128 tiles. In hundredths of a microsecond, measured at 8192^3, 4096^3, 94464 x 1364 x
// 1364, 5460 x 1364 x 2000, 2000 x 5460 x 1364 and 18750 x 6936 x 514: a round takes the longer of
// its copies (28 a block of 128 columns, 36 for a pair) and its epilogue (120, with slopes 400, a
// pair twice that), 60 more to fill and drain it, 120 for a pair, and a launch of pairs 400 more
// than one of single blocks. Single blocks and pairs: 8192^3 480 us and 305; 4096^3 67 and 45;
// 5460 x 1364 x 2000 23 and 17; 18750 x 6936 x 514 104 and 87; 1000 x 5460 x 1364 14.9 and 15.5;
// 93050 x 1075 x 88 89 and 98; 2000 x 5460 x 1364 with slopes 27 and 32.
bool use_pairs(const Params& p, int sms) {
  const int64_t pair_tiles = int64_t(p.tiles) / (int64_t(p.m_tiles) * p.n_tiles) * ((p.m_tiles + 1) / 2) * ((p.n_tiles + 1) / 2);
  const int64_t pairs = sms / 2, steps = int64_t(p.sum) * p.k_blocks, finish = p.slope ? 400 : 120;
  if (pairs < 1) return false;
  const int64_t one = steps * 28 > finish ? steps * 28 : finish, two = steps * 36 > 2 * finish ? steps * 36 : 2 * finish;
  return (pair_tiles + pairs - 1) / pairs * (two + 120) + 400 < (p.tiles + sms - 1) / sms * (one + 60);
}

}  // namespace

extern "C" emr_status emr_q8_matmul(const emr_q8* a, const emr_q8* w, const float* bias, int32_t act, int32_t sum_batch,
                                    void* out, int32_t out_dtype, const emr_q8* slope, void* stream) {
  if (!q8_ok(a) || !q8_ok(w) || a->cols != w->cols || !out || !dtype_ok(out_dtype) || act < EMR_ACT_IDENTITY ||
      act > EMR_ACT_ABS || (a->batch != w->batch && a->batch != 1 && w->batch != 1))
    return EMR_ERR_ARG;
  const int32_t batch = a->batch > w->batch ? a->batch : w->batch;
  if (sum_batch && (act != EMR_ACT_IDENTITY || bias || slope)) return EMR_ERR_ARG;
  if (slope && (!q8_ok(slope) || slope->batch != batch || slope->rows != a->rows || slope->cols != w->rows)) return EMR_ERR_ARG;
  const int size = dtype_bytes(out_dtype);
  if (reinterpret_cast<uintptr_t>(out) % size || (bias && reinterpret_cast<uintptr_t>(bias) % 4)) return EMR_ERR_ARG;
  Params p{};
  p.M = int32_t(a->rows), p.N = int32_t(w->rows);
  p.m_tiles = int32_t(q8_blocks(p.M)), p.n_tiles = int32_t(q8_blocks(p.N));
  const __int128 tiles = __int128(p.m_tiles) * p.n_tiles * (sum_batch ? 1 : batch);
  const __int128 steps = __int128(q8_blocks(a->cols)) * (sum_batch ? batch : 1);
  const int64_t reach = q8_row_bytes(a->cols) * (p.M > p.N ? p.M : p.N);  // bytes between two batches
  const int64_t scale_tiles = q8_scale_batch(p.M > p.N ? p.M : p.N, a->cols) / 512;
  if (tiles > INT32_MAX / 2 || steps > INT32_MAX || reach >= (int64_t(1) << 40) || __int128(scale_tiles) * batch > INT32_MAX)
    return EMR_ERR_RANGE;
  p.tiles = int32_t(tiles);
  p.k_blocks = int32_t(q8_blocks(a->cols)), p.k_chunks = int32_t(q8_scale_chunks(a->cols));
  p.sum = sum_batch ? batch : 1;
  p.a_one = a->batch == 1, p.w_one = w->batch == 1;
  p.a_scales = a->scales, p.w_scales = w->scales;
  p.bias = bias, p.act = act, p.out = out, p.out_dtype = out_dtype;
  p.store_bytes = 16;
  while (p.store_bytes > size && (reinterpret_cast<uintptr_t>(out) % p.store_bytes || (int64_t(p.N) * size) % p.store_bytes)) p.store_bytes >>= 1;
  p.narrow = !slope && p.N <= 64;
  if (slope) p.slope = slope->values, p.slope_scales = slope->scales, p.slope_whole = reinterpret_cast<uintptr_t>(slope->values) % 32 == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  if (!slope && use_thin(p, sms)) return launch_thin(a, w, p, dev, sms, st);
  CUtensorMap a_map, w_map;
  if (!operand_map(a, &a_map) || !operand_map(w, &w_map)) return EMR_ERR_CUDA;
  if (use_pairs(p, sms))
    return slope ? launch_pairs<true>(a, w, a_map, w_map, p, dev, sms, st) : launch_pairs<false>(a, w, a_map, w_map, p, dev, sms, st);
  return slope ? launch<true>(a_map, w_map, p, dev, sms, st) : launch<false>(a_map, w_map, p, dev, sms, st);
}

extern "C" emr_status emr_device_error(int32_t* code, void* stream) {
  if (!code) return EMR_ERR_ARG;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return first_record([&](int32_t* got) { return take_wait_error(g_wait_error, got, st); }, [&](int32_t* got) { return q4_wait_error(got, st); }, code);
}
