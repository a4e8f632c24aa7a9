// One index for each row of scores: temperature, top-k, top-p and min-p, and a draw by
// the largest w_i / noise_i, which is a draw from w when the noise is exponential (the
// smallest of exponentials of rates w_i belongs to i with probability w_i / sum w), so
// no running sum over the row is needed to draw.
//
// A row belongs to a cluster of 1 to 8 blocks, each with a slice of it in shared memory
// (kept in its own type) when that fits: scores are read from memory once. What top-k and
// top-p keep is a prefix of the order (score, larger first; index), so it is held as its
// last entry ("bound"). A histogram (counts, or sums of w) over (s_max - s) / T in equal
// steps finds the step in which the prefix ends; its entries are collected and ordered, or,
// where they are too many (rows with many equal scores), split again by the bytes of the
// score and at last by those of the index.
// Sums of w are integers (steps of 2^-F, F = 44 for rows up to 2^18, one less each time
// the row doubles after that), so that no result depends on the order of atomics.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "emr_q8.h"

namespace {

namespace cg = cooperative_groups;
using namespace emr;
typedef unsigned long long u64;

constexpr int kMaxThreads = 1024;
constexpr int kMaxCluster = 8;
constexpr float kSpan = 24.f;  // the equal steps cover w in (e^-24, 1]; the last one takes the rest

struct Args {
  const void* scores;
  int32_t dtype;
  int64_t n, row_stride, slice;  // slice: entries of one block
  const float* noise;
  int64_t noise_stride;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  float temperature_all, top_p_all, min_p_all;
  int32_t top_k_all;
  int32_t* index;
  float* logp;
  int32_t bins, cap;             // histogram steps, entries of the list
  int32_t resident, vector;      // slice kept in shared memory; 16-byte loads allowed
  int32_t fix;                   // F
};

// Order-preserving integer of a score that is not masked; masked ones give 0.
__device__ __forceinline__ uint32_t order_key(float s) {
  if (!(s > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(s + 0.f);  // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_score(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

struct Best {  // larger key first, then the lower index
  float key;
  int32_t at;
};
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.key > a.key || (b.key == a.key && uint32_t(b.at) < uint32_t(a.at)) ? b : a;
}

template <typename T>
struct Row {
  cg::cluster_group cluster;
  const Args& a;
  int tid, threads, lane, warp, warps, rank, blocks, phase;
  int64_t lo;       // first entry of this block's slice
  int count;        // its entries
  const T* global;  // the slice in memory
  T* data;          // and in shared memory
  uint32_t* counts;
  u64 *sums, *list, *sorted;
  u64* scratch;     // [64]
  u64* slots;       // [2][kMaxCluster]
  int* list_size;
  float s_max, temperature, min_w;

  __device__ __forceinline__ float get(int i) const { return float(a.resident ? data[i] : global[i]); }
  __device__ __forceinline__ float weight(float s) const {
    const float x = __fdiv_rn(s - s_max, temperature);
    return s == s_max ? 1.f : x <= 0.f ? expf(x) : 0.f;  // NaN: both infinite
  }
  __device__ __forceinline__ u64 fixed(float w) const { return __float2ull_rn(ldexpf(w, a.fix)); }
  __device__ __forceinline__ int step_of(float s, float per) const {
    const float t = (s_max - s) * per;  // falls as s rises; infinite and NaN (s_max infinite) go last or first
    return s == s_max ? 0 : t < float(a.bins - 1) ? int(t) : a.bins - 1;
  }
  __device__ void sync() {
    if (blocks > 1) cluster.sync();
    else __syncthreads();
  }
  // Reduction over the row's threads; every thread gets the result.
  template <typename V, typename Op>
  __device__ V reduce(V v, Op op) {
    static_assert(sizeof(V) == 8, "slots hold 8 bytes");
#pragma unroll
    for (int o = 16; o; o >>= 1) v = op(v, shfl_xor(v, o));
    __syncthreads();
    V* const part = reinterpret_cast<V*>(scratch);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < warps; i++) v = op(v, part[i]);
    if (blocks > 1) {
      V* const mine = reinterpret_cast<V*>(slots + phase * kMaxCluster);
      if (tid < blocks) *cluster.map_shared_rank(mine + rank, tid) = v;
      cluster.sync();
      v = mine[0];
      for (int i = 1; i < blocks; i++) v = op(v, mine[i]);
      phase ^= 1;  // a slot is written again only after the next reduction's barrier
    }
    return v;
  }
  template <typename V>
  __device__ __forceinline__ static V shfl_xor(V v, int o) {
    u64 u;
    memcpy(&u, &v, 8);
    u = __shfl_xor_sync(0xffffffffu, u, o);
    memcpy(&v, &u, 8);
    return v;
  }
  // Exclusive sum over the block's threads in order; *total gets the whole sum.
  __device__ u64 scan(u64 v, u64* total) {
    u64 in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 u = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += u;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = in;
    __syncthreads();
    u64 before = 0, all = 0;
    for (int i = 0; i < warps; i++) {
      if (i < warp) before += scratch[i];
      all += scratch[i];
    }
    *total = all;
    return before + in - v;
  }

  __device__ __forceinline__ bool kept(uint32_t key, int64_t at, uint32_t bound_key, int64_t bound_at) const {
    return key > bound_key || (key == bound_key && key != 0 && at <= bound_at);
  }

  // Entries for which `in(key, index)` holds, to the list of the row's first block (all of
  // them when they fit). Returns how many there are.
  template <typename In>
  __device__ int collect(In in) {
    if (tid == 0) *list_size = 0;
    sync();
    int* const size = blocks > 1 ? cluster.map_shared_rank(list_size, 0) : list_size;
    u64* const to = blocks > 1 ? cluster.map_shared_rank(list, 0) : list;
    for (int i = tid; i < count; i += threads) {
      const uint32_t key = order_key(get(i));
      if (key && in(key, lo + i)) {
        const int at = atomicAdd(size, 1);
        if (at < a.cap) to[at] = (u64(key) << 32) | uint32_t(~uint32_t(lo + i));
      }
    }
    sync();
    const int got = *size;
    sync();  // the size is read before it is set again
    return got;
  }
  // The list's m entries in order, in `sorted` of the row's first block: an entry's place
  // is the number of larger ones.
  __device__ void order(int m) {
    if (rank == 0)
      for (int j = tid; j < m; j += threads) {
        const u64 e = list[j];
        int place = 0;
        for (int i = 0; i < m; i++) place += list[i] > e;
        sorted[place] = e;
      }
    __syncthreads();
  }

  // Histogram of the entries `in` over `bins` steps `bin`, summed over the row, then the step in
  // which the wanted prefix ends: the last one before which less than the target lies. By count
  // (target entries) or by mass (p times the whole, when target is 0 it is p * whole).
  struct Found {
    int bin;
    int64_t size;    // entries of the step
    u64 before;      // entries, or mass, before it
    double target;
  };
  template <typename In, typename Bin>
  __device__ Found find(bool by_mass, int bins, double target, double p, In in, Bin bin, u64 base) {
    for (int i = tid; i < bins; i += threads) counts[i] = 0, sums[i] = 0;
    __syncthreads();
    for (int i = tid; i < count; i += threads) {
      const float s = get(i);
      const uint32_t key = order_key(s);
      if (key && in(key, lo + i)) {
        const int at = bin(s, key, lo + i);
        atomicAdd(&counts[at], 1u);
        if (by_mass) atomicAdd(&sums[at], fixed(weight(s)));
      }
    }
    sync();
    const int per = (bins + threads - 1) / threads;
    u64 mine = 0, total = 0;
    const int b0 = tid * per;
    auto value = [&](int b, bool mass) {
      u64 v = 0;
      for (int r = 0; r < blocks; r++) {
        const uint32_t* c = blocks > 1 ? cluster.map_shared_rank(counts, r) : counts;
        const u64* m = blocks > 1 ? cluster.map_shared_rank(sums, r) : sums;
        v += mass ? m[b] : c[b];
      }
      return v;
    };
    for (int b = b0; b < b0 + per && b < bins; b++) mine += value(b, by_mass);
    u64 before = base + scan(mine, &total);
    Found f{-1, 0, 0, target};
    if (by_mass && target < 0) f.target = fmax(double(total) * p, 0.5);  // one entry stays at least
    // the last step with entries that starts before the target
    u64 pick = 0;  // (bin + 1) of a candidate
    u64 pick_before = 0;
    int64_t pick_size = 0;
    for (int b = b0; b < b0 + per && b < bins; b++) {
      const u64 c = value(b, false), v = by_mass ? value(b, true) : c;
      if (c && double(before) < f.target) pick = u64(b) + 1, pick_before = before, pick_size = int64_t(c);
      before += v;
    }
    const u64 last = [&] {  // largest candidate of the block (every block sees the same)
      u64 v = pick;
      for (int o = 16; o; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
      __syncthreads();
      if (lane == 0) scratch[warp] = v;
      __syncthreads();
      v = scratch[0];
      for (int i = 1; i < warps; i++) v = max(v, scratch[i]);
      __syncthreads();
      return v;
    }();
    if (pick && pick == last) scratch[0] = pick_before, scratch[1] = u64(pick_size);
    __syncthreads();
    f.bin = int(last) - 1;
    f.before = scratch[0];
    f.size = last ? int64_t(scratch[1]) : 0;
    sync();  // histograms are read before they are cleared
    return f;
  }

  // Moves the bound (key, index) to the end of the prefix: `k` entries, or, by mass, the entries
  // before which less than p times the kept mass lies.
  __device__ void select(bool by_mass, int64_t k, double p, uint32_t& bound_key, int64_t& bound_at) {
    const uint32_t bk = bound_key;
    const int64_t ba = bound_at;
    const float per = float(a.bins - 1) / (kSpan * temperature);
    Found f = find(by_mass, a.bins, by_mass ? -1. : double(k), p, [&](uint32_t key, int64_t at) { return kept(key, at, bk, ba); },
                   [&](float s, uint32_t, int64_t) { return step_of(s, per); }, 0);
    const double target = f.target;
    const int step = f.bin;
    uint32_t prefix = 0;
    int shift = 32;  // key bits above `shift` are fixed to prefix
    auto in = [&](uint32_t key, int64_t at) {
      return kept(key, at, bk, ba) && (shift == 32 || (key >> shift) == prefix) && step_of(key_score(key), per) == step;
    };
    u64 before = f.before;
    int64_t size = f.size;
    while (size > a.cap && shift > 0) {
      const int next = shift - 8;
      // larger bytes first
      f = find(by_mass, 256, target, p, in, [&](float, uint32_t key, int64_t) { return 255 - int((key >> next) & 255u); }, before);
      prefix = (prefix << 8) | uint32_t(255 - f.bin);
      shift = next;
      before = f.before;
      size = f.size;
    }
    if (size <= a.cap) {
      const int m = collect(in);
      order(m);
      if (rank == 0) {
        if (!by_mass) {
          if (tid == 0) scratch[0] = sorted[int64_t(target) - int64_t(before) - 1];
        } else {
          // the last entry before which less than the target lies
          u64 run = before, found = 0;
          for (int j0 = 0; j0 < m; j0 += threads) {
            const int j = j0 + tid;
            u64 all;
            const u64 w = j < m ? fixed(weight(key_score(uint32_t(sorted[j] >> 32)))) : 0;
            const u64 ahead = run + scan(w, &all);
            if (j < m && double(ahead) < target) found = u64(j) + 1;
            run += all;
          }
          for (int o = 16; o; o >>= 1) found = max(found, __shfl_xor_sync(0xffffffffu, found, o));
          __syncthreads();
          if (lane == 0) scratch[warp] = found;
          __syncthreads();
          for (int i = 0; i < warps; i++) found = max(found, scratch[i]);
          __syncthreads();
          if (tid == 0) scratch[0] = sorted[found - 1];
        }
      }
      __syncthreads();
      u64 e = rank == 0 ? scratch[0] : 0;
      e = reduce(e, [](u64 x, u64 y) { return x > y ? x : y; });
      bound_key = uint32_t(e >> 32);
      bound_at = int64_t(uint32_t(~uint32_t(e)));
      return;
    }
    // equal scores: the first `want` of them by index
    const uint32_t key = prefix;
    int64_t want;
    if (!by_mass) want = int64_t(target) - int64_t(before);
    else {
      const u64 w = fixed(weight(key_score(key)));
      want = w == 0 ? size : int64_t(ceil((target - double(before)) / double(w)));
      want = want < 1 ? 1 : want > size ? size : want;
    }
    uint32_t ahead = 0;
    u64 passed = 0;
    for (int next = 24; next >= 0; next -= 8) {
      const int above = next + 8;
      const uint32_t fixed_bits = ahead;
      f = find(false, 256, double(want), p,
               [&](uint32_t x, int64_t at) { return x == key && at <= (x == bk ? ba : INT64_MAX) && (above == 32 || (uint32_t(at) >> above) == fixed_bits); },
               [&](float, uint32_t, int64_t at) { return int((uint32_t(at) >> next) & 255u); }, passed);
      ahead = (ahead << 8) | uint32_t(f.bin);
      passed = f.before;
    }
    bound_key = key;
    bound_at = int64_t(ahead);
  }

  // The draw over the kept entries: best w / noise, and the kept mass.
  __device__ void draw(const float* noise, uint32_t bound_key, int64_t bound_at, int32_t* index, float* logp) {
    Best best{-1.f, -1};
    u64 mass = 0;
    for (int i = tid; i < count; i += threads) {
      const float s = get(i);
      const uint32_t key = order_key(s);
      if (!kept(key, lo + i, bound_key, bound_at)) continue;
      const float w = weight(s);
      if (!(w >= min_w)) continue;
      mass += fixed(w);
      best = better(best, Best{w > 0.f ? __fdiv_rn(w, noise[lo + i]) : 0.f, int32_t(lo + i)});
    }
    finish(best, mass, index, logp);
  }
  __device__ void finish(Best best, u64 mass, int32_t* index, float* logp) {
    best = reduce(best, [](Best x, Best y) { return better(x, y); });
    mass = reduce(mass, [](u64 x, u64 y) { return x + y; });
    if (best.at < 0) {  // no positive noise among what stays
      if (rank == 0 && tid == 0) {
        *index = -1;
        if (logp) *logp = -INFINITY;
      }
    } else if (best.at >= lo && best.at < lo + count && tid == 0) {
      const float w = weight(get(int(best.at - lo)));
      *index = best.at;
      if (logp) *logp = float(log(double(w)) - log(ldexp(double(mass), -a.fix)));
    }
  }
};

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 1) sample_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ u64 scratch[64], slots[2 * kMaxCluster];
  __shared__ int list_size;
  Row<T> r{cg::this_cluster(), a};
  r.tid = threadIdx.x, r.threads = blockDim.x, r.lane = r.tid & 31, r.warp = r.tid >> 5, r.warps = r.threads >> 5;
  r.rank = int(r.cluster.block_rank()), r.blocks = int(r.cluster.num_blocks()), r.phase = 0;
  r.scratch = scratch, r.slots = slots, r.list_size = &list_size;
  r.sums = reinterpret_cast<u64*>(smem);
  r.counts = reinterpret_cast<uint32_t*>(r.sums + a.bins);
  r.sorted = r.sums;  // the histogram is done with when entries are ordered
  r.list = reinterpret_cast<u64*>(r.counts + a.bins);
  r.data = reinterpret_cast<T*>(r.list + a.cap);
  const int64_t row = blockIdx.x / unsigned(r.blocks);
  r.lo = r.rank * a.slice;
  r.count = int(a.n - r.lo < 0 ? 0 : a.n - r.lo < a.slice ? a.n - r.lo : a.slice);
  r.global = static_cast<const T*>(a.scores) + row * a.row_stride + r.lo;
  const float* noise = a.noise + row * a.noise_stride;
  int32_t* index = a.index + row;
  float* logp = a.logp ? a.logp + row : nullptr;

  float top = -INFINITY;
  constexpr int kPer = 16 / int(sizeof(T));
  int done = 0;
  if (a.vector) {
    for (int i = r.tid; i < r.count / kPer; i += r.threads) {
      const uint4 u = reinterpret_cast<const uint4*>(r.global)[i];
      if (a.resident) reinterpret_cast<uint4*>(r.data)[i] = u;
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < kPer; j++) top = fmaxf(top, float(e[j]));  // NaN is passed over
    }
    done = r.count / kPer * kPer;
  }
  for (int i = done + r.tid; i < r.count; i += r.threads) {
    const T e = r.global[i];
    if (a.resident) r.data[i] = e;
    top = fmaxf(top, float(e));
  }
  const uint32_t own_key = order_key(top);
  const u64 top_key = r.reduce(u64(own_key), [](u64 x, u64 y) { return x > y ? x : y; });
  if (top_key == 0) {  // nothing left
    if (r.rank == 0 && r.tid == 0) {
      *index = -1;
      if (logp) *logp = -INFINITY;
    }
    return;
  }
  r.s_max = key_score(uint32_t(top_key));
  r.temperature = a.temperature ? a.temperature[row] : a.temperature_all;
  r.min_w = fminf(a.min_p ? a.min_p[row] : a.min_p_all, 1.f);
  const int64_t k = a.top_k ? a.top_k[row] : a.top_k_all;
  const float p = a.top_p ? a.top_p[row] : a.top_p_all;

  if (!(r.temperature > 0.f)) {  // the largest score
    int64_t at = INT64_MAX;
    for (int i = r.tid; i < r.count; i += r.threads)
      if (r.get(i) == r.s_max) {
        at = r.lo + i;
        break;
      }
    at = r.reduce(at, [](int64_t x, int64_t y) { return x < y ? x : y; });
    if (r.rank == 0 && r.tid == 0) {
      *index = int32_t(at);
      if (logp) *logp = 0.f;
    }
    r.sync();
    return;
  }
  uint32_t bound_key = 0;
  int64_t bound_at = INT64_MAX;
  if (k > 0 && k < a.n) {
    // a score is masked or counted: fewer than k may be left, then all of them stay
    u64 valid = 0;
    for (int i = r.tid; i < r.count; i += r.threads) valid += order_key(r.get(i)) != 0;
    valid = r.reduce(valid, [](u64 x, u64 y) { return x + y; });
    if (u64(k) < valid) r.select(false, k, 0., bound_key, bound_at);
  }
  if (p < 1.f) r.select(true, 0, double(p), bound_key, bound_at);
  r.draw(noise, bound_key, bound_at, index, logp);
  r.sync();  // no block ends while another may still read its memory
}

template <typename T>
emr_status launch(const Args& a, int rows, int cluster, int threads, size_t smem, cudaStream_t st) {
  if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess)
    return EMR_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(rows) * unsigned(cluster));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = unsigned(cluster);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

}  // namespace

extern "C" emr_status emr_sample(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride,
                                 const float* noise, int64_t noise_stride, const float* temperature, float temperature_all,
                                 const int32_t* top_k, int32_t top_k_all, const float* top_p, float top_p_all,
                                 const float* min_p, float min_p_all, int32_t* index, float* logp, void* stream) {
  if (rows < 1 || n < 1 || !scores || !noise || !index || !dtype_ok(dtype) || row_stride < 0 || noise_stride < 0) return EMR_ERR_ARG;
  if (n > INT32_MAX || rows > (1 << 27)) return EMR_ERR_RANGE;
  const int size = dtype_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(scores) % size || reinterpret_cast<uintptr_t>(noise) % 4 ||
      reinterpret_cast<uintptr_t>(index) % 4 || reinterpret_cast<uintptr_t>(logp) % 4)
    return EMR_ERR_ARG;
  int dev = 0, sms = 0, room = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&room, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess)
    return EMR_ERR_CUDA;
  room -= 2048;  // the kernel's static arrays
  Args a{};
  a.scores = scores, a.dtype = dtype, a.n = n, a.row_stride = row_stride, a.noise = noise, a.noise_stride = noise_stride;
  a.temperature = temperature, a.top_k = top_k, a.top_p = top_p, a.min_p = min_p;
  a.temperature_all = temperature_all, a.top_k_all = top_k_all, a.top_p_all = top_p_all, a.min_p_all = min_p_all;
  a.index = index, a.logp = logp;
  int bits = 0;
  while ((int64_t(1) << bits) < n) bits++;
  a.fix = bits <= 18 ? 44 : 62 - bits;
  // Blocks of a row: as many as keep the device busy while a slice has 2048 entries, and as many
  // as a slice needs to fit into shared memory.
  int cluster = 1;
  while (cluster < kMaxCluster && int64_t(rows) * cluster * 2 <= sms && n / (cluster * 2) >= 2048) cluster *= 2;
  auto plan = [&] {
    a.slice = ((n + cluster - 1) / cluster + 15) / 16 * 16;
    const bool wide = a.slice > 8192;
    a.bins = wide ? 2048 : 512, a.cap = wide ? 2048 : 512;
    return size_t(a.bins) * 12 + size_t(a.cap) * 8;
  };
  size_t smem = plan();
  while (cluster < kMaxCluster && smem + size_t(a.slice) * size > size_t(room)) cluster *= 2, smem = plan();
  a.resident = smem + size_t(a.slice) * size <= size_t(room);
  if (a.resident) smem += size_t(a.slice) * size;
  a.vector = reinterpret_cast<uintptr_t>(scores) % 16 == 0 && (rows == 1 || (row_stride * size) % 16 == 0);
  const int threads = a.slice > 8192 ? 1024 : 256;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == EMR_F32) return launch<float>(a, rows, cluster, threads, smem, st);
  if (dtype == EMR_BF16) return launch<__nv_bfloat16>(a, rows, cluster, threads, smem, st);
  return launch<__half>(a, rows, cluster, threads, smem, st);
}
