// Barriers, copies and tensor-core access of the kernels that use tensor memory, each of them with its waits bounded.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/emr.h"

namespace {  // each translation unit has its own record of waits

// Number of a device-side wait that gave up (0: none); read by emr_device_error.
__device__ int g_wait_error = 0;
constexpr long long kWaitClocks = 4000000000ll;  // about 2 s

// ---- barriers and copies -----------------------------------------------------------

__device__ __forceinline__ uint32_t smem_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrivals of the epilogue: accumulators have been read into registers, which
// tcgen05.wait::ld and the fence before the arrival order. No store to memory is handed over, so
// they are relaxed: as releases they waited for the stores of the tile before (in a cluster's scope
// as far as L2: 18750 x 6936 x 514 141 us with, 87 without; 94464 x 1364 x 1364 161 and 140).
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// Waits for the phase; gives up after kWaitClocks, or as soon as another wait of the
// block has, and then records `code` once.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up, int code) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity)) {
    if (*gave_up) return false;
    if (clock64() - t0 > kWaitClocks) {
      *gave_up = code;
      atomicCAS(&g_wait_error, 0, code);
      return false;
    }
  }
  return true;
}
// The same by a whole warp, with one answer for it.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* gave_up, int code) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity, gave_up, code));
}
// One lane of a converged warp. The copy and matrix loops run in whole warps, whose addresses and
// descriptors then are uniform values, and only the instructions themselves belong to one lane:
// with the loops inside a branch of one lane each step took 690 clocks whatever it did.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// ---- tensor core -------------------------------------------------------------------

// Operand tile: rows of 128 bytes, swizzled by 128 bytes, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
  return uint64_t((addr & 0x3ffff) >> 4) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this warp's 32 accumulator rows: v[i] = column i of row `lane`.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; i++) v[i] = __uint_as_float(r[i]);
}

// After a wait gave up: longer than any copy or matrix instruction in flight takes.
__device__ __forceinline__ void settle() {
  const long long t0 = clock64();
  while (clock64() - t0 < 4000000) {
  }
}


// Place in the ring of stages: counted up, not divided, since the copy and matrix loops are
// one thread each and a block of 128 columns gives them 256 clocks.
template <int kCount>
struct Ring {
  int stage = 0;
  uint32_t round = 0;  // parity of the rounds made
  __device__ __forceinline__ void next() {
    if (++stage == kCount) stage = 0, round ^= 1;
  }
};

}  // namespace

namespace emr {

// The record of emr_q4_many.cu, and setting it back.
emr_status q4_wait_error(int32_t* code, cudaStream_t st);

// Reads a record and sets it back.
template <typename S>
emr_status take_wait_error(const S& symbol, int32_t* code, cudaStream_t st) {
  int32_t got = 0;
  const int32_t zero = 0;
  if (cudaMemcpyFromSymbolAsync(&got, symbol, 4, 0, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
    return EMR_ERR_CUDA;
  if (got && (cudaMemcpyToSymbolAsync(symbol, &zero, 4, 0, cudaMemcpyHostToDevice, st) != cudaSuccess ||
              cudaStreamSynchronize(st) != cudaSuccess))
    return EMR_ERR_CUDA;
  *code = got;
  return EMR_OK;
}

}  // namespace emr
