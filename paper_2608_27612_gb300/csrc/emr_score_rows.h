// One row of scores, or a slice of one, in the hands of a team of threads: what the kernels of log probabilities
// and of distillation share.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "emr_act.h"
#include "emr_q8.h"
#include "emr_rows.h"

namespace emr {
namespace rows {

namespace cg = cooperative_groups;

constexpr int kMaxCluster = 8;
constexpr float kFar = -1e4f;  // of d in units of log2: masked entries, whose w is 0 and w d too
constexpr float kLn2 = 0x1.62e43p-1f;

// The rows of a call.
struct Rows {
  const void* scores;
  int64_t n, row_stride, slice;  // slice: entries of one block
  int32_t rows;
  const float* temperature;
  float temperature_all;
  void* dscores;
  int64_t d_stride;
  int32_t d_dtype;
};

// Sums over some entries, with d = (s - m) / T in units of log2: of 2^d and of d 2^d.
struct Stat {
  float m, s, e;
};
// The same relative to a maximum that is no smaller.
__device__ __forceinline__ void shift(Stat& x, float m, float per) {
  const float d = x.m > -INFINITY ? fmaxf((x.m - m) * per, kFar) : 0.f, f = fast_exp2(d);
  x.e = f * fmaf(d, x.s, x.e), x.s *= f, x.m = m;
}
__device__ __forceinline__ void join(Stat& x, Stat y, float per) {
  const float m = fmaxf(x.m, y.m);
  shift(x, m, per), shift(y, m, per);
  x.s += y.s, x.e += y.e;
}
// x + v with the rounding kept in low.
__device__ __forceinline__ void add_kept(float& x, float& low, float v) {
  const float more = v - low, sum = x + more;
  low = (sum - x) - more, x = sum;
}

// One row, by a team of 32 threads (a warp of a block of 8) or of a block, and for a block's team by a cluster of them.
template <typename T, int kTeam>
struct Row {
  static constexpr int kG = Group<T>::kSize, kAhead = 4, kWarps = kTeam / 32;
  cg::cluster_group cluster;
  int tid, lane, warp, rank, blocks, phase, turn;
  int lo;            // first entry of this block's slice
  int count;         // its entries, the first of them `skip` entries after a multiple of 16 bytes
  int skip, groups;  // groups of 16 bytes that they lie in
  const T* global;   // the slice in memory
  uint4* scratch;    // [2][32], by turns: a turn's values are read by all before the next but one writes
  uint4* slots;      // [2][kMaxCluster]
  bool top_infinite; // only the entries of +infinity count, as score 0
  float per;         // log2(e) / T
  Stat own;          // of the thread's entries
  float s_low, e_low;

  __device__ Row(const Rows& a, int64_t row, uint4* scratch_, uint4* slots_) : cluster(cg::this_cluster()), scratch(scratch_), slots(slots_) {
    lane = threadIdx.x & 31;
    tid = kTeam == 32 ? lane : threadIdx.x;
    warp = tid >> 5;
    rank = kTeam == 32 ? 0 : int(cluster.block_rank()), blocks = kTeam == 32 ? 1 : int(cluster.num_blocks());
    phase = turn = 0;
    const int64_t at = rank * a.slice, left = a.n - at;
    lo = int(at < a.n ? at : a.n);
    count = int(left < 0 ? 0 : left < a.slice ? left : a.slice);
    global = static_cast<const T*>(a.scores) + row * a.row_stride + lo;
    skip = int(reinterpret_cast<uintptr_t>(global) % 16 / sizeof(T));
    groups = (skip + count + kG - 1) / kG;
    top_infinite = false;
  }
  __device__ __forceinline__ float value(T v) const {
    const float s = float(v);
    return top_infinite ? (s == INFINITY ? 0.f : -INFINITY) : s;
  }
  // One group from memory; past the slice its scores are -infinity.
  __device__ __forceinline__ Group<T> fetch(int g) const {
    Group<T> v;
    const int i = g * kG - skip;
    if (i >= 0 && i + kG <= count) {
      v.u = *reinterpret_cast<const uint4*>(global + i);
    } else {
#pragma unroll
      for (int j = 0; j < kG; j++) v.set(j, i + j >= 0 && i + j < count ? global[i + j] : T(-INFINITY));
    }
    return v;
  }
  __device__ __forceinline__ void floats(const Group<T>& v, float (&s)[kG]) const {
#pragma unroll
    for (int j = 0; j < kG; j++) s[j] = v.get(j);
    if (top_infinite) {
#pragma unroll
      for (int j = 0; j < kG; j++) s[j] = s[j] == INFINITY ? 0.f : -INFINITY;
    }
  }
  // fn(scores, g) for kAhead groups, loaded together: scores[u] is group g + u kTeam, -infinity past the slice. Of the
  // groups from first to before past, apart by whole turns.
  static constexpr int kTurn = kTeam * kAhead;
  template <typename Fn>
  __device__ __forceinline__ void each_group(Fn fn, int first, int past) const {
    for (int g = first + tid; g < past; g += kTurn) {
      Group<T> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; u++) v[u] = fetch(g + u * kTeam);
      float s[kAhead][kG];
#pragma unroll
      for (int u = 0; u < kAhead; u++) floats(v[u], s[u]);
      fn(s, g);
    }
  }

  template <typename Fn>
  __device__ __forceinline__ void each_group(Fn fn) const { each_group(fn, 0, groups); }

  __device__ __forceinline__ void team_sync() const {
    if (kTeam == 32) __syncwarp();
    else __syncthreads();
  }
  __device__ void row_sync() {
    if (blocks > 1) cluster.sync();
    else team_sync();
  }
  // One barrier for each of these: what a warp finds is combined by every warp again.
  __device__ uint32_t team_max(uint32_t v) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (kTeam == 32) return v;
    uint32_t* const part = reinterpret_cast<uint32_t*>(scratch + 32 * (turn ^= 1));
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < kWarps ? part[lane] : 0);
  }
  __device__ static float2 warp_sum(float2 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v.x += __shfl_xor_sync(0xffffffffu, v.x, o), v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    return v;
  }
  __device__ float2 team_sum(float2 v) {
    v = warp_sum(v);
    if (kTeam == 32) return v;
    float2* const part = reinterpret_cast<float2*>(scratch + 32 * (turn ^= 1));
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return warp_sum(lane < kWarps ? part[lane] : make_float2(0.f, 0.f));
  }
  // What every block has, to every block of the row: fn(value of block r), in the order of blocks.
  template <typename V, typename Fn>
  __device__ void exchange(const V& v, Fn fn) {
    static_assert(sizeof(V) <= 16, "slots hold 16 bytes");
    uint4* const mine = slots + phase * kMaxCluster;
    phase ^= 1;  // a slot is written again only after the next exchange's barrier
    if (tid < blocks) *reinterpret_cast<V*>(cluster.map_shared_rank(mine + rank, tid)) = v;
    cluster.sync();
    for (int i = 0; i < blocks; i++) fn(*reinterpret_cast<const V*>(mine + i));
  }

  // ---- sums --------------------------------------------------------------------------------

  __device__ __forceinline__ void begin() { own = {-INFINITY, 0.f, 0.f}, s_low = e_low = 0.f; }
  // kMean: also the sum of w d.
  template <bool kMean = true>
  __device__ __forceinline__ void add(const float (&s)[kAhead][kG]) {
    float most = s[0][0];
#pragma unroll
    for (int u = 0; u < kAhead; u++)
#pragma unroll
      for (int j = 0; j < kG; j++) most = fmaxf(most, s[u][j]);  // NaN is passed over
    if (most > own.m) {
      shift(own, most, per);
      s_low = e_low = 0.f;
    }
    if (own.m == -INFINITY) return;
    float w = 0.f, e = 0.f;
#pragma unroll
    for (int u = 0; u < kAhead; u++)
#pragma unroll
      for (int j = 0; j < kG; j++) {
        const float d = fmaxf((s[u][j] - own.m) * per, kFar), x = fast_exp2(d);  // the maximum takes NaN out, too
        w += x;
        if (kMean) e = fmaf(d, x, e);
      }
    add_kept(own.s, s_low, w);
    if (kMean) add_kept(own.e, e_low, e);
  }
  // The row's sums, of all threads' own.
  __device__ Stat total() {
    const uint32_t key = team_max(order_key(own.m));
    Stat all{key ? key_score(key) : -INFINITY, own.s, own.e};
    Stat mine = own;
    if (key) shift(mine, all.m, per);
    const float2 sum = team_sum(make_float2(mine.s, mine.e));
    all.s = sum.x, all.e = sum.y;
    if (blocks > 1) {
      const Stat part = all;
      all = {-INFINITY, 0.f, 0.f};
      exchange(part, [&](const Stat& x) {
        if (x.m > -INFINITY) join(all, x, per);
      });
    }
    return all;
  }

  // Where the row's largest score, m, stands first.
  __device__ int64_t first(float m) {
    uint32_t from_end = 0;
    each_group([&](const float (&s)[kAhead][kG], int g) {
#pragma unroll
      for (int u = 0; u < kAhead; u++)
#pragma unroll
        for (int j = 0; j < kG; j++)
          if (s[u][j] == m) from_end = max(from_end, 0xffffffffu - uint32_t(lo + (g + u * kTeam) * kG - skip + j));
    });
    from_end = team_max(from_end);
    if (blocks > 1) {
      const uint32_t part = from_end;
      exchange(part, [&](uint32_t x) { from_end = max(from_end, x); });
    }
    return 0xffffffffu - from_end;
  }

  // ---- the gradient --------------------------------------------------------------------------

  // Where the slice's gradient lies: pieces of up to 16 bytes where they are aligned as the scores' groups are.
  struct Out {
    uint8_t* p;
    int dtype, size;
    bool whole;
  };
  __device__ Out out(const Rows& a, int64_t row) const {
    Out o{static_cast<uint8_t*>(a.dscores), a.d_dtype, dtype_bytes(a.d_dtype), false};
    o.p += (row * a.d_stride + lo) * o.size;
    const int piece = kG * o.size < 16 ? kG * o.size : 16;
    o.whole = (reinterpret_cast<uintptr_t>(o.p) - uintptr_t(skip) * o.size) % piece == 0;
    return o;
  }
  template <typename D>
  __device__ __forceinline__ static void store_whole(uint8_t* p, const float (&v)[kG]) {
    constexpr int kBytes = kG * int(sizeof(D));
    uint32_t w[kBytes / 4];
    D* const d = reinterpret_cast<D*>(w);
#pragma unroll
    for (int j = 0; j < kG; j++) d[j] = D(v[j]);
    if (kBytes == 8) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
#pragma unroll
    for (int k = 0; k < kBytes / 16; k++)
      __stcs(reinterpret_cast<uint4*>(p) + k, make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]));
  }
  __device__ __forceinline__ void store(const Out& o, int g, const float (&v)[kG]) const {
    const int i = g * kG - skip;
    if (o.whole && i >= 0 && i + kG <= count) {
      uint8_t* const p = o.p + int64_t(i) * o.size;
      if (o.dtype == EMR_F32) store_whole<float>(p, v);
      else if (o.dtype == EMR_BF16) store_whole<__nv_bfloat16>(p, v);
      else store_whole<__half>(p, v);
    } else {
#pragma unroll
      for (int j = 0; j < kG; j++)
        if (i + j >= 0 && i + j < count) store_scalar(o.p, o.dtype, i + j, v[j]);
    }
  }
};

template <typename A>
emr_status launch_rows(void (*kernel)(A), const A& a, int team, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(team == 32 ? unsigned((int64_t(a.rows) + 7) / 8) : unsigned(a.rows) * unsigned(cluster));
  cfg.blockDim = dim3(team == 32 ? 256u : unsigned(team));
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = unsigned(cluster);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? EMR_OK : EMR_ERR_CUDA;
}

// How many clusters of each size run at the same time.
template <typename K>
void clusters_at_once(K kernel, int threads, int* fit) {
  for (int c = 1; c <= kMaxCluster; c++) {
    fit[c] = 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(c));
    cfg.blockDim = dim3(unsigned(threads));
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(c);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) fit[c] = n;
  }
}

// The team and cluster of a row, and the slice of its blocks. `wide`: what is asked for wants more threads than a warp.
inline int plan(Rows& a, bool wide, int sms, const int* fit, int* cluster) {
  *cluster = 1;
  a.slice = (a.n + 15) / 16 * 16;
  if (!wide && a.n <= 2048 && a.rows >= 8 * sms) return 32;
  if (a.n <= 8192) return 256;
  for (int c = 2; c <= kMaxCluster; c++)
    if (a.rows <= fit[c] && a.n / c >= 4096) *cluster = c;
  a.slice = ((a.n + *cluster - 1) / *cluster + 15) / 16 * 16;
  return 512;
}

inline bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline emr_status check_scores(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride) {
  if (rows < 1 || n < 1 || !scores || !dtype_ok(dtype) || row_stride < 0 || !aligned(scores, dtype_bytes(dtype))) return EMR_ERR_ARG;
  return n > INT32_MAX - (1 << 20) || rows > (1 << 27) ? EMR_ERR_RANGE : EMR_OK;
}

// Whether two arrays of so many elements share memory.
inline bool overlap(const void* x, int64_t nx, int size_x, const void* y, int64_t ny, int size_y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
  return a < b + uint64_t(ny) * size_y && b < a + uint64_t(nx) * size_x;
}

}  // namespace rows
}  // namespace emr
