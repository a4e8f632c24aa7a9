// Products of a few rows with 4-bit weights: y = act(x W^T + b), as a layer that serves single patterns wants them.
//
// y[m][n] = sum over groups g of scale[n][g] (sum over the group's k of code[n][k] x[m][k]): the inner sums are m16n8k16
// instructions with 16 rows of W as the instruction's rows and rows of x as its 8 columns, exact products with sums in 32
// bits, and each is scaled and added in 32 bits. Codes become 16-bit floats by one OR and one subtraction for two (128 + q as bfloat16,
// 1024 + q as float16). A 32-bit x is three bfloat16 parts of 8 bits each, together all of its 24 bits, in three columns.
// Bound by reading W: half a byte an entry and 2 / group for its scale, once for all columns, 48 at most (q4_is_many). x lies in shared memory, as
// much of a row as there is room for. A warp streams its units (16 rows x 128 columns, one piece of memory) into a
// ring of its own by asynchronous copies, five units ahead, and waits for no other warp. The warps of a block share rows of W
// (`wide`) or, where those are few, the contraction (`teams`); a cluster of up to 8 blocks shares the contraction of few
// rows further and adds its parts through distributed shared memory in the order of blocks. Where rows are many, a
// warp takes tile after tile.
// Measured on the device: 1 x 5460 x 1364 float32 7.2 us, 150 networks of 4 x 1364 x 256 float16 16.3 (32 MB, 2 TB/s; unpacking
// takes 40% of the instructions), 8 x 8192 x 8192 bfloat16 14.2 (36 MB, 2.5 TB/s, from HBM); x copied to registers by each warp,
// and warps that met after each unit, took 12.6, 31 and 23.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "emr_act.h"
#include "emr_q4.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;

constexpr int kThreads = 256, kWarps = kThreads / 32, kAhead = 6, kMaxCluster = 8;

struct Params {
  const uint8_t* w;
  int64_t w_batch;  // bytes of a matrix, 0 where all share it
  int32_t tiles, blocks;
  int64_t N, K, M;
  const void* x;
  int64_t x_batch, x_row, x_col;
  int32_t x_whole;     // 16 bytes of a row are one aligned piece
  int32_t wide, teams; // warps that share rows of W, and the contraction: powers of two
  int32_t log_teams;
  int32_t chunk;       // blocks of 128 columns whose x is in shared memory at a time
  int32_t row_blocks;  // blocks along the rows of a matrix, and all of them
  int32_t all_blocks;
  const float* bias;
  int32_t act;
  void* out;
  int32_t out_dtype;
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
// The first `bytes` of them, and zeros.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
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
// T: x. kN: tiles of 8 columns. kPer: groups in 128 columns.
template <typename T, int kN, int kPer>
__global__ void __launch_bounds__(kThreads, kN <= 2 ? 2 : 1) q4_few_kernel(const __grid_constant__ Params p) {
  constexpr bool kSplit = sizeof(T) == 4, kHalf = std::is_same<T, __half>::value;
  constexpr int kParts = kSplit ? 3 : 1;
  constexpr int kR = kN >= 4 ? 2 : 1;  // tiles of 16 rows of a warp, which share what is read of x
  constexpr int kUnit = kQ4Codes + 32 * kPer, kStage = kR * kUnit;
  extern __shared__ __align__(16) uint8_t smem[];
  const auto cluster = cg::this_cluster();
  const int shares = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int wide = p.wide, teams = p.teams, in_rows = warp & (wide - 1), team = warp >> (3 - p.log_teams);
  const int rows = int(p.M), columns = kParts * rows;
  const int first = shares == 1 ? 0 : int(unsigned(p.blocks) * unsigned(rank) / unsigned(shares));
  const int last = shares == 1 ? p.blocks : int(unsigned(p.blocks) * unsigned(rank + 1) / unsigned(shares));
  // blocks of rows of the block, one after the other
  const unsigned here = shares == 1 ? blockIdx.x : blockIdx.x / unsigned(shares), grid = shares == 1 ? gridDim.x : gridDim.x / unsigned(shares);
  const int from = int(grid == unsigned(p.all_blocks) ? here : unsigned(uint64_t(p.all_blocks) * here / grid));
  const int past = int(grid == unsigned(p.all_blocks) ? here + 1 : unsigned(uint64_t(p.all_blocks) * (here + 1) / grid));

  const int pitch = p.chunk * 256 + 64;  // of a column of x, in bytes: its 16-bit values, and other banks than the one before
  uint8_t* const ring = smem + warp * (kAhead * kStage);
  uint8_t* const xs = smem + kWarps * kAhead * kStage;
  const uint32_t ring_at = uint32_t(__cvta_generic_to_shared(ring)) + lane * 16, xs_at = uint32_t(__cvta_generic_to_shared(xs));

  // the warp's part of the chunk that begins with block c: of teams as many
  const auto part_of = [&](int c, int team) { return c + ((last - c < p.chunk ? last - c : p.chunk) * team >> p.log_teams); };
  // The stream of its units, by blocks of rows, chunks and blocks of columns.
  int s_block = from, s_b = p.row_blocks == p.all_blocks ? 0 : from / p.row_blocks, s_row = from - s_b * p.row_blocks;
  const int s_first_b = s_b;
  int s_chunk = first, s_kb = 0, s_end = 0, s_stage = 0, s_tiles = 0;
  const uint8_t* s_unit = nullptr;
  const auto seek = [&] {  // to the next part that is not empty
    while (s_kb == s_end && s_block < past) {
      const int tile = (s_row * wide + in_rows) * kR;
      s_tiles = p.tiles - tile;
      s_kb = part_of(s_chunk, team), s_end = s_tiles > 0 ? part_of(s_chunk, team + 1) : s_kb;
      s_unit = p.w + s_b * p.w_batch + (int64_t(tile) * p.blocks + s_kb) * kUnit + lane * 16;
      s_chunk += p.chunk;
      if (s_chunk >= last) {
        s_chunk = first, s_block++;
        if (++s_row == p.row_blocks) s_row = 0, s_b++;
      }
    }
  };
  const auto issue = [&] {
    if (s_kb < s_end) {
#pragma unroll
      for (int r = 0; r < kR; r++) {
        if (r && r >= s_tiles) break;
        const uint8_t* const unit = s_unit + int64_t(r) * p.blocks * kUnit;
        const uint32_t to = ring_at + s_stage * kStage + r * kUnit;
        copy16(to, unit);
        copy16(to + 512, unit + 512);
        if (lane < 2 * kPer) copy16(to + kQ4Codes, unit + kQ4Codes);
      }
      s_stage = s_stage == kAhead - 1 ? 0 : s_stage + 1;
      s_unit += kUnit;
      if (++s_kb == s_end) seek();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  seek();
#pragma unroll 1
  for (int i = 0; i < kAhead - 1; i++) issue();

  // x of a chunk: a thread's pieces of 16 bytes, as they lie or, if that cannot be, four at a time through registers
  const auto stage_x = [&](int b, int c) {
    constexpr int kPiece = kSplit ? 4 : 8;
    const int per_row = (last - c < p.chunk ? last - c : p.chunk) * (kQ4Cols / kPiece);
    const int64_t k0 = int64_t(c) * kQ4Cols;
    const T* const x = static_cast<const T*>(p.x) + b * p.x_batch + k0 * p.x_col;
    const int log_rows = rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0, apart = 32 << (3 - log_rows);  // warps of a row: 8, 4, 2 or 1
    for (int m = warp & ((1 << log_rows) - 1); m < rows; m += 1 << log_rows) {
      const T* const row = x + m * p.x_row;
      const int have = int(p.K - k0 < int64_t(per_row) * kPiece ? p.K - k0 : int64_t(per_row) * kPiece);
      int i = lane + (warp >> log_rows) * 32;
      if (!kSplit && p.x_whole) {
        uint32_t to = xs_at + m * pitch + i * 16;
        for (; i < per_row; i += apart, to += apart * 16) {
          const int left = have - i * 8;
          copy16(to, left > 0 ? row + i * 8 : row, left >= 8 ? 16 : left > 0 ? left * 2 : 0);
        }
        continue;
      }
#pragma unroll 1
      for (; i < per_row; i += 4 * apart) {
        uint4 piece[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const int at = (i + u * apart) * kPiece, left = have - at;
          const T* const from = row + at * p.x_col;
          if (p.x_whole && left >= kPiece) {
            piece[u] = *reinterpret_cast<const uint4*>(from);
          } else {
            T* const v = reinterpret_cast<T*>(piece + u);
#pragma unroll
            for (int j = 0; j < kPiece; j++) v[j] = j < left ? from[j * p.x_col] : T(0.f);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; u++) {
          if (i + u * apart >= per_row) break;
          uint8_t* const to = xs + m * pitch + (i + u * apart) * (kPiece * 2);
          if constexpr (kSplit) {
            uint2 part[3];
            split_pair(__uint_as_float(piece[u].x), __uint_as_float(piece[u].y), part[0].x, part[1].x, part[2].x);
            split_pair(__uint_as_float(piece[u].z), __uint_as_float(piece[u].w), part[0].y, part[1].y, part[2].y);
#pragma unroll
            for (int q = 0; q < 3; q++) *reinterpret_cast<uint2*>(to + q * rows * pitch) = part[q];
          } else {
            *reinterpret_cast<uint4*>(to) = piece[u];
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
  };

  float sum[kR][kN][4];
  const auto clear = [&] {
#pragma unroll
    for (int r = 0; r < kR; r++)
#pragma unroll
      for (int n = 0; n < kN; n++)
#pragma unroll
        for (int j = 0; j < 4; j++) sum[r][n][j] = 0.f;
  };
  clear();
  // Output (m, n0 + n) of matrix b, at `at` + m N + n, from what `of` gives for its columns.
  const auto finish = [&](int b, int64_t n0, int64_t at, int m, int n, auto of) {
    if (n0 + n >= p.N) return;
    float z[1] = {of(m)}, d[1];
#pragma unroll
    for (int c = 1; c < kParts; c++) z[0] += of(c * rows + m);
    if (p.bias) z[0] += p.bias[b * p.N + n0 + n];
    activate<1, false>(p.act, z, d);
    store_scalar(p.out, p.out_dtype, at + m * p.N + n, z[0]);
  };
  // A warp's sums: [column][row].
  float* const own = reinterpret_cast<float*>(xs + columns * pitch) + warp * (kR * kN * 128);

  int stage = 0;
  int64_t staged = -1;  // whose x is there
  int b = s_first_b, row_block = from - b * p.row_blocks;
  for (int block = from; block < past; block++) {
    const int tile = (row_block * wide + in_rows) * kR;
    for (int c = first; c < last; c += p.chunk) {
      const int64_t wanted = (p.x_batch ? int64_t(b) * p.blocks : 0) + c;
      if (wanted != staged) {
        if (staged >= 0) __syncthreads();
        stage_x(b, c);
        __syncthreads();
        staged = wanted;
      }
      const int end = tile < p.tiles ? part_of(c, team + 1) : 0;
      for (int kb = part_of(c, team); kb < end; kb++) {
        issue();
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        __syncwarp();
        const uint8_t* const unit = ring + stage * kStage;
        const uint8_t* const e_from = xs + (kb - c) * 256 + t * 16 + g * pitch;
        stage = stage == kAhead - 1 ? 0 : stage + 1;
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
        for (int q = 0; q < kPer; q++) {
          constexpr int kChains = kN == 1 ? 2 : 1;  // sums that do not wait for one another
          float part[kChains][kR][kN][4];
#pragma unroll
          for (int h = 0; h < kChains; h++)
#pragma unroll
            for (int r = 0; r < kR; r++)
#pragma unroll
              for (int n = 0; n < kN; n++)
#pragma unroll
                for (int j = 0; j < 4; j++) part[h][r][n][j] = 0.f;
#pragma unroll
          for (int v = q * (4 / kPer); v < (q + 1) * (4 / kPer); v++) {  // 32 columns: two steps of 16
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
              if (n * 8 + g < columns) e = *reinterpret_cast<const uint4*>(e_from + v * 64 + n * 8 * pitch);
#pragma unroll
              for (int r = 0; r < kR; r++) {
                mma<kHalf>(part[0][r][n], a[0][r], e.x, e.y);
                mma<kHalf>(part[kChains - 1][r][n], a[1][r], e.z, e.w);
              }
            }
          }
#pragma unroll
          for (int r = 0; r < kR; r++)
#pragma unroll
            for (int n = 0; n < kN; n++)
#pragma unroll
              for (int j = 0; j < 4; j++) {
                const float all = kChains == 2 ? part[0][r][n][j] + part[kChains - 1][r][n][j] : part[0][r][n][j];
                sum[r][n][j] = fmaf(scale[r][(j >> 1) * kPer + q], all, sum[r][n][j]);
              }
        }
        __syncwarp();
      }
    }
    if (teams == 1 && shares == 1 && tile < p.tiles) {  // a warp's own outputs
#pragma unroll
      for (int r = 0; r < kR; r++)
#pragma unroll
        for (int n = 0; n < kN; n++)
#pragma unroll
          for (int j = 0; j < 4; j++) own[(n * 8 + 2 * t + (j & 1)) * (kR * 16) + r * 16 + g + 8 * (j >> 1)] = sum[r][n][j];
      __syncwarp();
      const int64_t n0 = int64_t(tile) * 16, at = b * p.M * p.N + n0;
      for (int i = lane; i < rows * kR * 16; i += 32) {
        const int n = i % (kR * 16);
        finish(b, n0, at, i / (kR * 16), n, [&](int column) { return own[column * (kR * 16) + n]; });
      }
      __syncwarp();
      clear();
    }
    if (++row_block == p.row_blocks) row_block = 0, b++;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (teams == 1 && shares == 1) return;

  // one block of rows: the warps' sums, [team][column][row of the block]; then those of the blocks of the cluster
  __syncthreads();
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
  const int64_t n0 = int64_t(from - s_first_b * p.row_blocks) * tall, out_at = s_first_b * p.M * p.N + n0;
  const int log_tall = __ffs(tall) - 1;
  if (shares > 1) {
    for (int at = tid; at < columns * tall; at += kThreads) {
      float v = sums[at];
      for (int i = 1; i < teams; i++) v += sums[i * room + at];
      sums[at] = v;
    }
    cluster.sync();
    for (int at = rank * kThreads + tid; at < rows * tall; at += kThreads * shares) {
      const int n = at & (tall - 1);
      finish(s_first_b, n0, out_at, at >> log_tall, n, [&](int column) {
        float v = 0.f;
        for (int i = 0; i < shares; i++) v += cluster.map_shared_rank(sums, i)[column * tall + n];
        return v;
      });
    }
    cluster.sync();  // a block's sums are read by the others
  } else {
    for (int at = tid; at < rows * tall; at += kThreads) {
      const int n = at & (tall - 1);
      finish(s_first_b, n0, out_at, at >> log_tall, n, [&](int column) {
        float v = 0.f;
        for (int i = 0; i < teams; i++) v += sums[i * room + column * tall + n];
        return v;
      });
    }
  }
}

template <typename T, int kN, int kPer>
emr_status launch(const Params& p, int64_t blocks, int shares, size_t smem, int dev, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(q4_few_kernel<T, kN, kPer>, kMostSmem, dev, done)) return EMR_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(blocks * shares));
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
  const int columns = int(p.M) * kParts, kn = columns <= 8 ? 1 : columns <= 16 ? 2 : columns <= 32 ? 4 : 8, kr = kn >= 4 ? 2 : 1;
  const int64_t row_tiles = (p.tiles + kr - 1) / kr;
  const size_t unit = kQ4Codes + 32 * per, ring = size_t(kWarps) * kAhead * kr * unit, sums = size_t(kWarps) * kr * 16 * kn * 8 * 4;
  // x: beside the rings, in half an SM's shared memory where two blocks share it
  const size_t most = kn <= 2 ? 110 * 1024 : kMostSmem, room = most - ring;
  const int fit = int((room - columns * 64) / (size_t(columns) * 256)), fit_direct = int((room - sums - columns * 64) / (size_t(columns) * 256));
  int64_t blocks;
  int shares = 1;
  if (p.blocks <= fit_direct && batch * row_tiles >= kWarps * sms) {
    // enough tiles for every warp of an SM: each takes its own, two blocks an SM
    p.wide = kWarps, p.teams = 1, p.chunk = p.blocks;
    p.row_blocks = int((row_tiles + kWarps - 1) / kWarps);
    const int64_t all = batch * p.row_blocks;
    if (all > INT32_MAX) return EMR_ERR_RANGE;
    p.all_blocks = int32_t(all);
    const int64_t room_for = (kn <= 2 ? 2 : 1) * sms;
    blocks = p.all_blocks < room_for ? p.all_blocks : room_for;
  } else {
    // every block reads x: rows of W enough that x is at most half as many bytes, and that its share of x fits at once
    int wide = 1;
    while (wide < kWarps && int(p.M) * int(sizeof(T)) > wide * kr * 4) wide *= 2;
    const int at_once = (kn <= 2 ? 2 : 1) * sms;
    for (;; wide *= 2) {
      p.wide = wide, p.teams = kWarps / wide;
      p.row_blocks = int((row_tiles + wide - 1) / wide);
      blocks = batch * p.row_blocks;
      shares = 1;
      for (int s = 2; s <= kMaxCluster; s++)
        if (blocks * s <= at_once && p.blocks / (s * p.teams) >= 2) shares = s;
      const int share = (p.blocks + shares - 1) / shares, some = p.teams == 1 ? fit_direct : fit, parts = (share + some - 1) / some;
      p.chunk = (share + parts - 1) / parts;
      if (parts == 1 || wide == kWarps) break;
    }
    if (blocks > INT32_MAX) return EMR_ERR_RANGE;
    p.all_blocks = int32_t(blocks);
  }
  if (blocks * shares > INT32_MAX) return EMR_ERR_RANGE;
  for (p.log_teams = 0; (1 << p.log_teams) < p.teams;) p.log_teams++;
  const bool own = p.teams == 1 && shares == 1;
  size_t smem = ring + size_t(columns) * (p.chunk * 256 + 64) + (own ? sums : 0);
  if (smem < sums) smem = sums;
  if constexpr (kParts == 3) {  // 16-bit rows, 32 at most, are no more columns
    if (kn == 8) return launch<T, 8>(p, per, blocks, shares, smem, dev, st);
  }
  return kn == 1   ? launch<T, 1>(p, per, blocks, shares, smem, dev, st)
         : kn == 2 ? launch<T, 2>(p, per, blocks, shares, smem, dev, st) : launch<T, 4>(p, per, blocks, shares, smem, dev, st);
}

// The arguments of a product, checked.
emr_status describe(const void* x, int32_t dtype, int32_t x_batch, int64_t rows, int64_t batch_stride, int64_t row_stride, int64_t col_stride,
                    const emr_q4* w, emr::Q4Product* a) {
  if (!q4_ok(w) || !x || rows < 1 || x_batch < 1 || (x_batch != 1 && w->batch != 1 && x_batch != w->batch) || !dtype_ok(dtype) ||
      batch_stride < 0 || row_stride < 0 || col_stride < 0 || reinterpret_cast<uintptr_t>(x) % dtype_bytes(dtype))
    return EMR_ERR_ARG;
  size_t bytes;
  const emr_status ok = emr_q4_size(w->batch, w->rows, w->cols, w->group, &bytes);
  if (ok != EMR_OK) return ok;
  if (rows > kQ8MaxDim) return EMR_ERR_RANGE;
  const int piece = 16 / dtype_bytes(dtype);
  *a = {w, x, dtype, x_batch, rows, batch_stride, row_stride, col_stride, false, nullptr, 0, nullptr, 0};
  a->whole = col_stride == 1 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && (rows == 1 || row_stride % piece == 0) &&
             (x_batch == 1 || batch_stride % piece == 0);
  return double(x_batch) * double(rows) * double(w->cols) > 1e17 ? EMR_ERR_RANGE : EMR_OK;
}

}  // namespace

extern "C" emr_status emr_q4_matmul_room(const void* x, int32_t dtype, int32_t x_batch, int64_t rows, int64_t batch_stride, int64_t row_stride,
                                         int64_t col_stride, const emr_q4* w, size_t* bytes) {
  emr::Q4Product a;
  if (!bytes) return EMR_ERR_ARG;
  const emr_status ok = describe(x, dtype, x_batch, rows, batch_stride, row_stride, col_stride, w, &a);
  if (ok == EMR_OK) *bytes = emr::q4_is_many(a) ? emr::q4_many_room(a) : 0;
  return ok;
}

extern "C" emr_status emr_q4_matmul(const void* x, int32_t dtype, int32_t x_batch, int64_t rows, int64_t batch_stride, int64_t row_stride,
                                    int64_t col_stride, const emr_q4* w, const float* bias, int32_t act, void* out, int32_t out_dtype, void* ws,
                                    size_t ws_bytes, void* stream) {
  emr::Q4Product a;
  const emr_status ok = describe(x, dtype, x_batch, rows, batch_stride, row_stride, col_stride, w, &a);
  if (ok != EMR_OK) return ok;
  if (!out || !dtype_ok(out_dtype) || act < EMR_ACT_IDENTITY || act > EMR_ACT_ABS || reinterpret_cast<uintptr_t>(out) % dtype_bytes(out_dtype) ||
      reinterpret_cast<uintptr_t>(bias) % 4)
    return EMR_ERR_ARG;
  const int64_t batch = x_batch > w->batch ? x_batch : w->batch;
  if (overlap(x, (x_batch - 1) * batch_stride + (rows - 1) * row_stride + (w->cols - 1) * col_stride + 1, dtype_bytes(dtype), out, batch * rows * w->rows,
              dtype_bytes(out_dtype)) ||
      overlap(w->data, w->batch * q4_tiles(w->rows) * q4_blocks(w->cols) * q4_unit(w->group), 1, out, batch * rows * w->rows, dtype_bytes(out_dtype)) ||
      (bias && overlap(bias, batch * w->rows, 4, out, batch * rows * w->rows, dtype_bytes(out_dtype))))  // read by other rows after one is written
    return EMR_ERR_ARG;
  a.bias = bias, a.act = act, a.out = out, a.out_dtype = out_dtype;
  int dev = 0, sms = 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (emr::q4_is_many(a)) {
    const size_t room = emr::q4_many_room(a);
    if (room && (!ws || reinterpret_cast<uintptr_t>(ws) % 16)) return EMR_ERR_ARG;
    if (ws_bytes < room) return EMR_ERR_CAPACITY;
    return device_sms(&dev, &sms) ? emr::launch_q4_many(a, ws, dev, sms, st) : EMR_ERR_CUDA;
  }
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  Params p{};
  p.w = w->data, p.tiles = int32_t(q4_tiles(w->rows)), p.blocks = int32_t(q4_blocks(w->cols));
  p.w_batch = w->batch == 1 ? 0 : int64_t(p.tiles) * p.blocks * q4_unit(w->group);
  p.N = w->rows, p.K = w->cols, p.M = rows;
  p.x = x, p.x_batch = x_batch == 1 ? 0 : batch_stride, p.x_row = row_stride, p.x_col = col_stride, p.x_whole = a.whole;
  p.bias = bias, p.act = act, p.out = out, p.out_dtype = out_dtype;
  const int per = kQ4Cols / w->group;
  if (dtype == EMR_F32) return plan<float>(p, batch, per, dev, sms, st);
  if (dtype == EMR_BF16) return plan<__nv_bfloat16>(p, batch, per, dev, sms, st);
  return plan<__half>(p, batch, per, dev, sms, st);
}
