// Block-scaled 8-bit matrices: quantising, transposing, reading back, and the
// backward pass of an activation from its 8-bit slope.
//
// Every kernel reads its source once: a row block of 128 columns is one warp's
// registers (four columns a lane, or sixteen of eight lanes), so its maximum is one
// reduction over lanes and its codes one 128-byte store; the transposed copy is made
// from the same registers through a 16 KB tile of codes. Bytes are the floor; by rows
// 8192 x 8192 bfloat16 takes 33 us (6.1 TB/s), 94464 x 1364 float16 72 (5.5). The tiles of
// both ways are bound by the instructions of the reductions and conversions (ALU pipe
// 65%, memory 40%): 64 us (4.2 TB/s), the slope product with sums 93 (3.6).
#include <cuda_runtime.h>

#include "emr_q8.h"

namespace {

using namespace emr;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kTileThreads = 512;

// Dense source. kRows: columns are neighbours; kFours: and every row is aligned to four elements.
enum Layout { kStrided, kRows, kFours };
template <typename T, Layout kLayout>
struct Dense {
  using Value = T;
  static constexpr bool kWhole = kLayout != kStrided;  // rows lie in one piece
  const T* p;
  int64_t batch_stride, row_stride, col_stride;
};

__device__ __forceinline__ float4 q8_four(const uint8_t* values, const uint8_t* scales, int64_t row_bytes,
                                          int64_t chunks, int64_t r, int64_t c) {
  const float s = q8_scale(scales[q8_scale_at(chunks, r, c >> 7)]);
  const float4 v = q8_unpack4(*reinterpret_cast<const uint32_t*>(values + r * row_bytes + c));
  return make_float4(v.x * s, v.y * s, v.z * s, v.w * s);
}

// An address that copies of no bytes may name.
__device__ __forceinline__ const void* aligned_down(const void* p) {
  return reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15));
}
// 4, 8 or 16 bytes from memory into shared memory, past `have` bytes zeros.
template <int kBytes>
__device__ __forceinline__ void copy_ahead(void* to, const void* from, int have) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(uint32_t(__cvta_generic_to_shared(to))), "l"(from), "n"(kBytes),
               "r"(have)
               : "memory");
}

// Row blocks only, of rows that lie in one piece. Eight lanes have a block, sixteen columns each, so
// that what is done once for a block is done once for sixteen values of a lane. Blocks are a grid's
// groups of eight apart; a lane copies those of its next turns into shared memory of its own in
// aligned units of 16 bytes, out of which a row that starts elsewhere is shifted. What a unit holds
// besides the row is not used, and nothing is read from outside the matrix. Addresses are counted up:
// with them computed for every block the kernel was bound by its integer instructions (8192 x 8192
// bfloat16 47 us, now 33).
template <typename T>
struct Rows16 {
  static constexpr int kUnits = int(sizeof(T)) + 1;
  static constexpr int kAhead = 2;  // turns
  static constexpr int kSmem = (kAhead + 1) * kUnits * kThreads * 16;
  static constexpr int kBlocks = sizeof(T) == 4 ? 3 : 5;  // of an SM
};
// Indices of blocks fit 32 bits: 2^32 of them are more than a device holds.
template <typename T, bool kBatch>
__global__ void __launch_bounds__(kThreads, Rows16<T>::kBlocks)
    q8_rows16_kernel(const T* src, const T* last, int64_t batch_stride, int64_t row_stride, uint32_t rows, uint32_t blocks, int32_t tail,
                     uint32_t all, emr_q8 q) {
  constexpr int kUnits = Rows16<T>::kUnits, kAhead = Rows16<T>::kAhead;
  extern __shared__ __align__(16) uint4 ring[];  // [turn][unit][thread]
  const int lane = threadIdx.x & 31, part = (lane & 7) * 16;
  const uint32_t stride = gridDim.x * kWarps * 4, far_rows = stride / blocks, far_blocks = stride - far_rows * blocks;
  const int64_t scale_batch = q8_scale_batch(rows, int64_t(blocks) * 128);
  const uint32_t chunks = (blocks + 3) / 4;
  const int tail_cells = tail - part;  // of this lane in a row's last block
  uint32_t g = (blockIdx.x * kWarps + (threadIdx.x >> 5)) * 4 + (lane >> 3), row = g / blocks, kb = g - row * blocks;
  // the copies run kAhead turns before: block, and its address where it follows from the one before
  uint32_t next_g = g, next_row = row, next_kb = kb, turn = 0, shifts = 0;
  const T* at = src + int64_t(row) * row_stride + int64_t(kb) * 128 + part;
  const int64_t step = int64_t(far_rows) * row_stride + int64_t(far_blocks) * 128, wrap = row_stride - int64_t(blocks) * 128;
  const auto copy = [&] {
    if (kBatch) {
      const uint32_t b = next_row / rows;
      at = src + int64_t(b) * batch_stride + int64_t(next_row - b * rows) * row_stride + int64_t(next_kb) * 128 + part;
    }
    const uint32_t shift = uint32_t(reinterpret_cast<uintptr_t>(at)) & 15;
    shifts = shifts << 4 | shift;
    if (next_g < all && (next_kb + 1 < blocks || tail_cells > 0)) {
      uint4* const to = ring + turn * (kUnits * kThreads) + threadIdx.x;
      const char* const unit = reinterpret_cast<const char*>(at) - shift;
      if (unit >= reinterpret_cast<const char*>(src) && unit + kUnits * 16 <= reinterpret_cast<const char*>(last)) {
#pragma unroll
        for (int i = 0; i < kUnits; i++)
          if (i + 1 < kUnits || shift) copy_ahead<16>(to + i * kThreads, unit + i * 16, 16);
      } else {  // at the matrix's ends
#pragma unroll
        for (int i = 0; i < kUnits; i++) {
#pragma unroll
          for (int e = 0; e < 16; e += int(sizeof(T))) {
            const T* const from = reinterpret_cast<const T*>(unit + i * 16 + e);
            *reinterpret_cast<T*>(reinterpret_cast<char*>(to + i * kThreads) + e) = from >= src && from < last ? *from : T(0.f);
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    next_g += stride, next_row += far_rows, next_kb += far_blocks, at += step;
    if (next_kb >= blocks) next_kb -= blocks, next_row++, at += wrap;
    turn = turn == kAhead ? 0 : turn + 1;
  };
  grid_wait();
  grid_go();
#pragma unroll
  for (int i = 0; i < kAhead; i++) copy();
  uint8_t* out = q.values + int64_t(g) * 128 + part;
  uint32_t own = 0;
  while (__any_sync(0xffffffffu, g < all)) {
    copy();
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
    uint32_t w[kUnits * 4];
#pragma unroll
    for (int i = 0; i < kUnits; i++)
      *reinterpret_cast<uint4*>(w + 4 * i) = ring[(own * kUnits + i) * kThreads + threadIdx.x];
    const uint32_t shift = shifts >> (4 * kAhead) & 15;
    if (shift) {
#pragma unroll
      for (int i = 0; i < kUnits * 4 - 2; i++) w[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
      for (int i = 0; i < kUnits * 4 - 3; i++) w[i] = shift & 4 ? w[i + 1] : w[i];
      if (sizeof(T) == 2) {
        const uint32_t select = shift & 2 ? 0x5432 : 0x3210;
#pragma unroll
        for (int i = 0; i < kUnits * 4 - 4; i++) w[i] = __byte_perm(w[i], w[i + 1], select);
      }
    }
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = float(reinterpret_cast<const T*>(w)[i]);
    const int cells = g >= all ? 0 : kb + 1 < blocks ? 16 : tail_cells;
    if (cells < 16) {
#pragma unroll
      for (int i = 0; i < 16; i++) v[i] = i < cells ? v[i] : 0.f;
    }
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) most = fmaxf(most, fabsf(v[i]));
    uint32_t top = __float_as_uint(most);  // NaN is passed over
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 4));
    if (__any_sync(0xffffffffu, top >= 0x7f800000u)) {  // an infinity: finite magnitudes again
      top = 0;
#pragma unroll
      for (int i = 0; i < 16; i++) top = max(top, q8_magnitude(v[i])), v[i] = q8_finite_or_nan(v[i]);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 4));
    }
    const uint32_t byte = q8_scale_byte(top);
    const float inv = q8_inverse(byte);
    if (g < all) {
      *reinterpret_cast<uint4*>(out) = make_uint4(q8_pack4(v[0], v[1], v[2], v[3], inv), q8_pack4(v[4], v[5], v[6], v[7], inv),
                                                  q8_pack4(v[8], v[9], v[10], v[11], inv), q8_pack4(v[12], v[13], v[14], v[15], inv));
      if (part == 0) {
        const uint32_t b = kBatch ? row / rows : 0, r = row - b * rows;
        q.scales[(kBatch ? b * scale_batch : 0) + (int64_t(r >> 7) * chunks + (kb >> 2)) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4 + (kb & 3)] =
            uint8_t(byte);
      }
    }
    g += stride, out += int64_t(stride) * 128, row += far_rows, kb += far_blocks;
    if (kb >= blocks) kb -= blocks, row++;
    own = own == kAhead ? 0 : own + 1;
  }
}

// 128 x 128 tiles: row blocks to q, column blocks (the transpose) to qt, column sums to
// sums[b][row tile][cols]. Mode 0: a dense source; 1: the values of an 8-bit matrix; 2: the
// product of a dense matrix and an 8-bit one; 3: a dense source whose transpose is made of
// the values that q holds. A block goes through tiles gridDim.x apart
// and copies the next one into shared memory while it works on one; of the dense source a
// thread reads back only what it copied itself. A warp holds the rows 8 warp .. 8 warp + 7 in registers, a
// lane four columns of each. Column maxima and sums meet in shared memory over the 16
// warps (the sums in their order); codes of four rows are one word of the transposed byte
// tile, at (row / 4) ^ (column / 4 % 32) of its column, so that neither the stores (lanes:
// columns 4 apart) nor the loads (lanes: one column) have conflicts.
template <int kMode, typename T, Layout kLayout>
__global__ void __launch_bounds__(kTileThreads, 2) q8_tile_kernel(Dense<T, kLayout> src, emr_q8 other, int64_t rows, int64_t cols,
                                                                  uint32_t tiles, emr_q8 q, emr_q8 qt, float* sums) {
  constexpr bool kFromQ8 = kMode == 1 || kMode == 2;
  constexpr bool kPieces = kMode != 1 && kLayout == kRows && sizeof(T) == 2;
  constexpr int kPitch = 17 * 16 + 16;  // of a row in pieces; the last 16 bytes are only read along
  extern __shared__ __align__(16) uint8_t ahead[];  // [8][threads] of the dense source, then two tiles of codes
  __shared__ float4 part[16][32];
  __shared__ uint32_t bytes[128 * 32];
  __shared__ uint32_t tops[2][4][32];  // by turns: [j][lane], largest magnitude of column 4 lane + j
  const uint32_t row_tiles = uint32_t(q8_blocks(rows)), col_tiles = uint32_t(q8_blocks(cols));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp * 8;
  const int64_t chunks = q8_scale_chunks(cols), row_bytes = q8_row_bytes(cols), scale_batch = q8_scale_batch(rows, cols);
  const int64_t t_row_bytes = q8_row_bytes(rows), t_chunks = q8_scale_chunks(rows), t_scale_batch = q8_scale_batch(cols, rows);
  Four<T>* const dense = reinterpret_cast<Four<T>*>(ahead) + threadIdx.x;
  uint8_t* const rows_ahead = ahead + first * kPitch;
  uint8_t* const codes = ahead + (kPieces ? 128 * kPitch : kMode != 1 ? sizeof(Four<T>) * 8 * kTileThreads : 0);

  struct Place {
    int64_t b, rt, ct;
    int have, wide;  // rows of this warp (may be below 1) and columns of the tile
  };
  const auto place = [&](uint32_t t) {
    Place p;
    const uint32_t rest = t / col_tiles;
    p.ct = t - rest * col_tiles;
    const uint32_t b = rest / row_tiles;
    p.b = b, p.rt = rest - b * row_tiles;
    const int64_t left = rows - p.rt * 128, right = cols - p.ct * 128;
    p.have = int(left < 128 ? left : 128) - first;
    p.wide = int(right < 128 ? right : 128);
    return p;
  };
  uint32_t next_scale = 127;
  const auto copy = [&](const Place& p, uint32_t turn) {
    const int64_t c = p.ct * 128 + lane * 4;
    if (kMode != 1) {
      const int n = p.wide - lane * 4, cells = n < 0 ? 0 : n < 4 ? n : 4;
      const T* from = src.p + p.b * src.batch_stride + (p.rt * 128 + first) * src.row_stride;
      if constexpr (kPieces) {
        // two-byte elements at any address: a warp copies its rows in aligned pieces of 16 bytes, 17 of
        // which hold a row's 128 elements, and reads them back shifted
#pragma unroll
        for (int k = 0; k < 5; k++) {
          const int piece = lane + k * 32, i = piece / 17, at = (piece - i * 17) * 16;
          if (piece >= 8 * 17) break;
          const char* row = reinterpret_cast<const char*>(from + i * src.row_stride + p.ct * 128);
          const char* piece_from = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(15)) + at;
          uint8_t* to = rows_ahead + i * kPitch + at;
          const int64_t left = row + p.wide * 2 - piece_from;
          if (i < p.have && piece_from < reinterpret_cast<const char*>(src.p)) {  // nothing is read from before the matrix
#pragma unroll
            for (int e = 0; e < 16; e += 2)
              *reinterpret_cast<uint16_t*>(to + e) =
                  piece_from + e >= row && e < left ? *reinterpret_cast<const uint16_t*>(piece_from + e) : uint16_t(0);
          } else {
            const int have = i >= p.have || left <= 0 ? 0 : left < 16 ? int(left) : 16;
            copy_ahead<16>(to, have ? static_cast<const void*>(piece_from) : aligned_down(src.p), have);
          }
        }
      }
      const bool inner = p.have >= 8 && p.wide == 128;
      const T* row = from + c;
#pragma unroll
      for (int i = 0; i < (kPieces ? 0 : 8); i++) {
        if constexpr (kLayout == kRows && sizeof(T) == 4) {
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const bool in = i < p.have && j < cells;
            copy_ahead<4>(reinterpret_cast<uint32_t*>(dense + i * kTileThreads) + j, in ? from + i * src.row_stride + c + j : src.p, in ? 4 : 0);
          }
        } else if constexpr (kLayout == kFours) {
          if (inner) {
            copy_ahead<int(sizeof(Four<T>))>(dense + i * kTileThreads, row, int(sizeof(Four<T>)));
            row += src.row_stride;
            continue;
          }
          const bool in = i < p.have && cells > 0;
          copy_ahead<int(sizeof(Four<T>))>(dense + i * kTileThreads, in ? from + i * src.row_stride + c : src.p, in ? cells * int(sizeof(T)) : 0);
        } else {
          Four<T> u;
#pragma unroll
          for (int j = 0; j < 4; j++) u.set(j, i < p.have && j < cells ? from[i * src.row_stride + (c + j) * src.col_stride] : T(0.f));
          dense[i * kTileThreads] = u;
        }
      }
    }
    if (kFromQ8) {
      // 16 bytes a thread, to be read by other threads
      const uint8_t* from = other.values + (p.b * rows + p.rt * 128) * row_bytes + p.ct * 128;
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int r = (threadIdx.x >> 3) + i * 64, at = (threadIdx.x & 7) * 16;
        const bool in = r < p.have + first;
        copy_ahead<16>(codes + turn * 16384 + r * 128 + at, in ? from + r * row_bytes + at : other.values, in ? 16 : 0);
      }
      next_scale = 127;
      if (lane < 8 && lane < p.have) next_scale = other.scales[p.b * scale_batch + q8_scale_at(chunks, p.rt * 128 + first + lane, p.ct)];
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  if (threadIdx.x < 256) (&tops[0][0][0])[threadIdx.x] = 0;
  grid_wait();
  grid_go();
  Place p = place(blockIdx.x), after = p;
  copy(p, 0);
  __syncthreads();
  uint32_t turn = 0;
  for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x, turn ^= 1, p = after) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (kFromQ8) __syncthreads();
    else if (kPieces) __syncwarp();
    float4 v[8];
    const uint32_t scale_bytes = next_scale;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      if constexpr (kPieces) {
        const uintptr_t start = reinterpret_cast<uintptr_t>(src.p + p.b * src.batch_stride + (p.rt * 128 + first + i) * src.row_stride + p.ct * 128);
        const int at = int(start & 15) + lane * 8;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(rows_ahead + i * kPitch + (at & ~3));
        Four<T> u;
        u.u = make_uint2(w[0], w[1]);
        if (start & 2) u.u = make_uint2(__funnelshift_r(u.u.x, u.u.y, 16), __funnelshift_r(u.u.y, w[2], 16));
        const int cells = p.wide - lane * 4;  // what lies after the row in its last piece is not of it
        if (cells < 4) {
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (j >= cells) u.set(j, T(0.f));
        }
        v[i] = i < p.have ? u.floats() : make_float4(0.f, 0.f, 0.f, 0.f);
      } else if constexpr (kMode != 1) {
        v[i] = dense[i * kTileThreads].floats();
      }
      if (kFromQ8) {
        const float s = q8_scale(__shfl_sync(0xffffffffu, scale_bytes, i));
        float4 d = q8_unpack4(*reinterpret_cast<const uint32_t*>(codes + turn * 16384 + (first + i) * 128 + lane * 4));
        d = make_float4(d.x * s, d.y * s, d.z * s, d.w * s);
        // one rounding each, so that the values are those of the plain product
        v[i] = kMode == 1 ? d : make_float4(__fmul_rn(v[i].x, d.x), __fmul_rn(v[i].y, d.y), __fmul_rn(v[i].z, d.z), __fmul_rn(v[i].w, d.w));
      }
    }
    if (kPieces) __syncwarp();  // the rows are read before others take their place
    if (t + gridDim.x < tiles) after = place(t + gridDim.x), copy(after, turn ^ 1);
    if (sums) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; i++) s.x += v[i].x, s.y += v[i].y, s.z += v[i].z, s.w += v[i].w;
      part[warp][lane] = s;
      __syncthreads();
      if (int(threadIdx.x) < p.wide) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i++) sum += reinterpret_cast<const float*>(part[i])[threadIdx.x];
        sums[(p.b * row_tiles + p.rt) * cols + p.ct * 128 + threadIdx.x] = sum;
      }
    }
    if (q.values) {
      uint8_t* out = q.values + (p.b * rows + p.rt * 128 + first) * row_bytes + p.ct * 128 + lane * 4;
      // lane i has the largest magnitude of row i, so that all eight scales are made at once (8192 x
      // 8192 bfloat16 both ways 70 us with one after the other, 64 so)
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(q8_top4(v[i])));
        most = lane == i ? top : most;
      }
      if (__any_sync(0xffffffffu, most >= 0x7f800000u)) {  // an infinity, or nothing but NaN in some lane
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(q8_magnitude(v[i].x), q8_magnitude(v[i].y)),
                                                                  max(q8_magnitude(v[i].z), q8_magnitude(v[i].w))));
          most = lane == i ? top : most;
          v[i] = make_float4(q8_finite_or_nan(v[i].x), q8_finite_or_nan(v[i].y), q8_finite_or_nan(v[i].z), q8_finite_or_nan(v[i].w));
        }
      }
      const uint32_t mine = q8_scale_byte(most);
      const float mine_inv = q8_inverse(mine);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint32_t codes4 = q8_pack4(v[i].x, v[i].y, v[i].z, v[i].w, __shfl_sync(0xffffffffu, mine_inv, i));
        if (i < p.have) *reinterpret_cast<uint32_t*>(out) = codes4;
        if (kMode == 3) {
          const float4 d = q8_unpack4(codes4);
          const float s = q8_scale(__shfl_sync(0xffffffffu, mine, i));
          v[i] = make_float4(d.x * s, d.y * s, d.z * s, d.w * s);
        }
        out += row_bytes;
      }
      if (lane < 8 && lane < p.have) q.scales[p.b * scale_batch + q8_scale_at(chunks, p.rt * 128 + first + lane, p.ct)] = uint8_t(mine);
    }
    if (!qt.values) {
      if (sums) __syncthreads();  // the sums are read before the next ones are written
      continue;
    }
    float4 top = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; i++)
      top = make_float4(fmaxf(top.x, fabsf(v[i].x)), fmaxf(top.y, fabsf(v[i].y)), fmaxf(top.z, fabsf(v[i].z)), fmaxf(top.w, fabsf(v[i].w)));
    // NaN is passed over by the maxima; where an infinity is, the finite magnitudes are taken again
    if (q8_top4(top) == INFINITY) {
      if constexpr (kMode == 1 || kMode == 3) {
        // codes stand for no infinity: it is 2^128, as which values from 1.9375 * 2^127 on are held and which
        // 32 bits do not have. The largest of them is held as the same.
        const auto held = [](float f) { return fabsf(f) == INFINITY ? copysignf(__uint_as_float(0x7f7fffffu), f) : f; };
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = make_float4(held(v[i].x), held(v[i].y), held(v[i].z), held(v[i].w));
      }
      uint32_t m[4] = {};
#pragma unroll
      for (int i = 0; i < 8; i++) {
        m[0] = max(m[0], q8_magnitude(v[i].x)), m[1] = max(m[1], q8_magnitude(v[i].y));
        m[2] = max(m[2], q8_magnitude(v[i].z)), m[3] = max(m[3], q8_magnitude(v[i].w));
        v[i] = make_float4(q8_finite_or_nan(v[i].x), q8_finite_or_nan(v[i].y), q8_finite_or_nan(v[i].z), q8_finite_or_nan(v[i].w));
      }
      top = make_float4(__uint_as_float(m[0]), __uint_as_float(m[1]), __uint_as_float(m[2]), __uint_as_float(m[3]));
    }
    atomicMax(&tops[turn][0][lane], __float_as_uint(top.x));
    atomicMax(&tops[turn][1][lane], __float_as_uint(top.y));
    atomicMax(&tops[turn][2][lane], __float_as_uint(top.z));
    atomicMax(&tops[turn][3][lane], __float_as_uint(top.w));
    __syncthreads();
    const uint32_t scale[4] = {q8_scale_byte(tops[turn][0][lane]), q8_scale_byte(tops[turn][1][lane]), q8_scale_byte(tops[turn][2][lane]),
                               q8_scale_byte(tops[turn][3][lane])};
    const float inv[4] = {q8_inverse(scale[0]), q8_inverse(scale[1]), q8_inverse(scale[2]), q8_inverse(scale[3])};
    if (warp == 0) {
      uint8_t* ts = qt.scales + p.b * t_scale_batch;
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (lane * 4 + j < p.wide) ts[q8_scale_at(t_chunks, p.ct * 128 + lane * 4 + j, p.rt)] = uint8_t(scale[j]);
    }
    if (warp < 4) tops[turn ^ 1][warp][lane] = 0;  // read by all before the barrier above
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int w = (warp * 2 + h) ^ lane;  // word of rows first + 4 h ..., columns 4 lane + j
      bytes[(lane * 4 + 0) * 32 + w] = q8_pack4(v[4 * h].x, v[4 * h + 1].x, v[4 * h + 2].x, v[4 * h + 3].x, inv[0]);
      bytes[(lane * 4 + 1) * 32 + w] = q8_pack4(v[4 * h].y, v[4 * h + 1].y, v[4 * h + 2].y, v[4 * h + 3].y, inv[1]);
      bytes[(lane * 4 + 2) * 32 + w] = q8_pack4(v[4 * h].z, v[4 * h + 1].z, v[4 * h + 2].z, v[4 * h + 3].z, inv[2]);
      bytes[(lane * 4 + 3) * 32 + w] = q8_pack4(v[4 * h].w, v[4 * h + 1].w, v[4 * h + 2].w, v[4 * h + 3].w, inv[3]);
    }
    __syncthreads();
    uint8_t* out = qt.values + (p.b * cols + p.ct * 128 + first) * t_row_bytes + p.rt * 128 + lane * 4;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int n = first + i;
      if (n < p.wide) *reinterpret_cast<uint32_t*>(out) = bytes[n * 32 + (lane ^ (n >> 2))];
      out += t_row_bytes;
    }
  }
}

// Sum of the row tiles' column sums, in the order of the tiles.
__global__ void __launch_bounds__(kThreads) q8_sums_kernel(const float* sums, int64_t row_tiles, int64_t cols,
                                                           int64_t total, void* db, int dtype) {
  grid_wait();
  grid_go();
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

template <int kMode, typename T, Layout kLayout>
emr_status launch_tile(const Dense<T, kLayout>& src, const emr_q8* other, int64_t batch, int64_t rows, int64_t cols,
                       const emr_q8* q, const emr_q8* qt, float* sums, cudaStream_t st) {
  const int64_t tiles = batch * q8_blocks(rows) * q8_blocks(cols);
  if (tiles > kMaxGrid) return EMR_ERR_RANGE;
  static std::atomic<uint64_t> done{0};
  const bool pieces = kMode != 1 && kLayout == kRows && sizeof(T) == 2;
  const int smem = (pieces ? 128 * 288 : kMode != 1 ? int(sizeof(Four<T>)) * 8 * kTileThreads : 0) + (kMode == 1 || kMode == 2 ? 2 * 16384 : 0);
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms) || !allow_smem(q8_tile_kernel<kMode, T, kLayout>, smem, dev, done)) return EMR_ERR_CUDA;
  const emr_q8 none{};
  return launch_after(q8_tile_kernel<kMode, T, kLayout>, dim3(unsigned(tiles < 2 * sms ? tiles : 2 * sms)), kTileThreads, size_t(smem), st,
                      src, other ? *other : none, rows, cols, uint32_t(tiles), q ? *q : none, qt ? *qt : none, sums);
}

template <typename T, bool kBatch>
emr_status launch_rows16(const T* p, int64_t batch_stride, int64_t row_stride, int64_t batch, int64_t rows, int64_t cols, const emr_q8* q,
                         cudaStream_t st) {
  const int64_t blocks = q8_blocks(cols);
  const __int128 all = __int128(batch) * rows * blocks;
  int dev = 0, sms = 0;
  if (!device_sms(&dev, &sms)) return EMR_ERR_CUDA;
  const int64_t most = int64_t(sms) * Rows16<T>::kBlocks;
  if (all > UINT32_MAX - 4 * most * kWarps * 4) return EMR_ERR_RANGE;
  const int64_t need = (int64_t(all) + kWarps * 4 - 1) / (kWarps * 4);
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(q8_rows16_kernel<T, kBatch>, Rows16<T>::kSmem, dev, done)) return EMR_ERR_CUDA;
  return launch_after(q8_rows16_kernel<T, kBatch>, dim3(unsigned(need < most ? need : most)), kThreads, size_t(Rows16<T>::kSmem), st, p,
                      p + (batch - 1) * batch_stride + (rows - 1) * row_stride + cols, batch_stride, row_stride, uint32_t(rows),
                      uint32_t(blocks), int32_t(cols - (blocks - 1) * 128), uint32_t(all), *q);
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
  if (vector) return fn(Dense<T, kFours>{p, a.batch_stride, a.row_stride, a.col_stride});
  if (a.col_stride == 1) return fn(Dense<T, kRows>{p, a.batch_stride, a.row_stride, 1});
  return fn(Dense<T, kStrided>{p, a.batch_stride, a.row_stride, a.col_stride});
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
    if constexpr (d.kWhole) {
      if (!qt && batch == 1) return launch_rows16<typename decltype(d)::Value, false>(d.p, 0, d.row_stride, 1, rows, cols, q, st);
      if (!qt) return launch_rows16<typename decltype(d)::Value, true>(d.p, d.batch_stride, d.row_stride, batch, rows, cols, q, st);
    }
    return launch_tile<0>(d, nullptr, batch, rows, cols, q, qt, nullptr, st);
  });
}

extern "C" emr_status emr_q8_quantize_held(const void* src, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                                           int64_t batch_stride, int64_t row_stride, int64_t col_stride, const emr_q8* q,
                                           const emr_q8* qt, void* stream) {
  if (!src || !dtype_ok(dtype) || batch < 1 || rows < 1 || cols < 1 || batch_stride < 0 || row_stride < 0 || col_stride < 0)
    return EMR_ERR_ARG;
  if (rows > kQ8MaxDim || cols > kQ8MaxDim) return EMR_ERR_RANGE;
  if (!same_shape(q, batch, rows, cols) || !same_shape(qt, batch, cols, rows) || reinterpret_cast<uintptr_t>(src) % dtype_bytes(dtype))
    return EMR_ERR_ARG;
  const DenseArgs args{src, dtype, batch, rows, cols, batch_stride, row_stride, col_stride};
  return with_dense(args, [&](auto d) {
    return launch_tile<3>(d, nullptr, batch, rows, cols, q, qt, nullptr, static_cast<cudaStream_t>(stream));
  });
}

extern "C" emr_status emr_q8_transpose(const emr_q8* q, const emr_q8* qt, void* stream) {
  if (!q8_ok(q) || !same_shape(qt, q->batch, q->cols, q->rows)) return EMR_ERR_ARG;
  return launch_tile<1>(Dense<float, kFours>{}, q, q->batch, q->rows, q->cols, nullptr, qt, nullptr,
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
  return launch_after(q8_sums_kernel, dim3(unsigned(grid)), kThreads, 0, st, sums, q8_blocks(rows), cols, total, db, db_dtype);
}
