// One row of scores, or a slice of one, in the hands of a team of threads: what the kernels of log probabilities
// and of distillation share.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// Two values at a time.
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 c, a, b;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 c, a, b;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
  return r;
}
// (s - m) / T of two scores in units of log2, masked ones at kFar: the maximum takes NaN out, too.
__device__ __forceinline__ float2 far2(float s0, float s1, float m, float per) {
  const float2 d = mul2(add2(make_float2(s0, s1), make_float2(-m, -m)), make_float2(per, per));
  return make_float2(fmaxf(d.x, kFar), fmaxf(d.y, kFar));
}

// One row, by a team of 8 or 32 threads (of a block of 256) or of a block of 64 to 512, and for the largest team by a cluster of blocks.
// Threads take it in turns of kAhead groups of 16 bytes each, loaded together and without a check, while all threads have as
// many; the groups that are left, among them those that reach out of the slice, one at a time.
template <typename T, int kTeam>
struct Row {
  static constexpr int kG = Group<T>::kSize, kAhead = 4, kWarps = kTeam < 32 ? 1 : kTeam / 32, kTurn = kTeam * kAhead, kTeamSize = kTeam;
  cg::cluster_group cluster;
  int tid, lane, warp, rank, blocks, phase, turn;
  int lo;            // first entry of this block's slice
  int count;         // its entries, the first of them `skip` entries after a multiple of 16 bytes
  int skip, groups;  // groups of 16 bytes that they lie in
  int head;          // 1 where the first of them reaches out of the slice
  const T* global;   // the slice in memory
  bool inside;       // the rest of its first and last group lies in the scores' memory, too
  uint4* scratch;    // [2][32], by turns: a turn's values are read by all before the next but one writes
  uint4* slots;      // [2][kMaxCluster]
  bool asks;         // in a cluster's first pass of two: for the turn after the next, in L2, by one instruction while a turn is read
                     // (gradients of 512 x 87380 float32 79 -> 73 us, distillation of 1000 x 87380 float16 84 -> 78; the best answers gain nothing)
  bool top_infinite; // only the entries of +infinity count, as score 0
  float per;         // log2(e) / T
  Stat own;          // of the thread's entries
  float s_low, e_low;

  __device__ __forceinline__ Row(const Rows& a, int64_t row, uint4* scratch_, uint4* slots_) : cluster(cg::this_cluster()), scratch(scratch_), slots(slots_) {
    lane = threadIdx.x & (kTeam < 32 ? kTeam - 1 : 31);
    tid = kTeam <= 32 ? lane : threadIdx.x;
    warp = tid >> 5;
    rank = kTeam < 512 ? 0 : int(cluster.block_rank()), blocks = kTeam < 512 ? 1 : int(cluster.num_blocks());
    phase = turn = 0;
    const int64_t at = rank * a.slice, left = a.n - at;
    lo = int(at < a.n ? at : a.n);
    count = int(left < 0 ? 0 : left < a.slice ? left : a.slice);
    const T* const scores = static_cast<const T*>(a.scores);
    global = scores + row * a.row_stride + lo;
    skip = int(reinterpret_cast<uintptr_t>(global) % 16 / sizeof(T));
    groups = (skip + count + kG - 1) / kG;
    inside = global - skip >= scores && global - skip + int64_t(groups) * kG <= scores + (a.rows - 1) * a.row_stride + a.n;
    top_infinite = asks = false;
    head = skip ? 1 : 0;
  }
  __device__ __forceinline__ float value(T v) const {
    const float s = float(v);
    return top_infinite ? (s == INFINITY ? 0.f : -INFINITY) : s;
  }
  // One group from memory, which may reach out of the slice.
  __device__ __forceinline__ Group<T> fetch(int g) const {
    const int i = g * kG - skip;
    Group<T> v;
    if (!inside && (i < 0 || i + kG > count)) v.u = fetch_part(global, i, count);
    else v.u = *reinterpret_cast<const uint4*>(global + i);
    return v;
  }
  // Asks for the slice's first groups, 128 bytes for each thread, while something else is read.
  __device__ __forceinline__ void ahead() const {
    if (tid * (128 / int(sizeof(T))) < count) asm volatile("prefetch.global.L2 [%0];" ::"l"(global + tid * (128 / int(sizeof(T)))));
  }
  // The same where what lies around the scores may not be read.
  __device__ static __noinline__ uint4 fetch_part(const T* global, int i, int count) {
    Group<T> v;
#pragma unroll
    for (int j = 0; j < kG; j++) v.set(j, unsigned(i + j) < unsigned(count) ? global[i + j] : T(0.f));
    return v.u;
  }
  // With a score of +infinity in the row all others do not count.
  __device__ __forceinline__ void infinite(Group<T>& v) const {
#pragma unroll
    for (int j = 0; j < kG; j++) v.set(j, v.get(j) == INFINITY ? T(0.f) : T(-INFINITY));
  }
  // One group, -infinity out of the slice.
  __device__ __forceinline__ Group<T> masked(int g) const {
    Group<T> v = fetch(g);
    const int i = g * kG - skip;
    if (i < 0 || i + kG > count) {
#pragma unroll
      for (int j = 0; j < kG; j++)
        if (unsigned(i + j) >= unsigned(count)) v.mask(j);
    }
    if (top_infinite) infinite(v);
    return v;
  }
  __device__ __forceinline__ static void floats(const Group<T>& v, float (&s)[kG]) {
#pragma unroll
    for (int j = 0; j < kG; j++) s[j] = v.get(j);
  }
  // fn(v, g) of an array of groups g, g + kTeam ... that lie in the slice as a whole, or of one group, for those from first
  // (head or more) to before past, and the first one of all where with_head: after the others.
  template <int kN, typename Fn>
  __device__ __forceinline__ void turn_of(Fn& fn, int& g, const uint4*& from) const {
    Group<T> v[kN];
#pragma unroll
    for (int u = 0; u < kN; u++) v[u].u = from[u * kTeam];
    if (top_infinite) {
#pragma unroll
      for (int u = 0; u < kN; u++) infinite(v[u]);
    }
    fn(v, g);
    g += kN * kTeam, from += kN * kTeam;
  }
  template <typename Fn>
  __device__ __forceinline__ void each(Fn& fn, int first, int past, bool with_head) const {
    const int whole = (skip + count) / kG < past ? (skip + count) / kG : past, turns = (whole - first) / kTurn;
    int g = first + tid;
    const uint4* from = reinterpret_cast<const uint4*>(global + (g * kG - skip));
    const int all = (skip + count) / kG;
    for (int i = 0; i < turns; i++) {
      const int at = first + (i + 2) * kTurn;
      if (kTeam == 512 && asks && tid == 0 && at < all)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(global + (int64_t(at) * kG - skip)), "r"((all - at < kTurn ? all - at : kTurn) * 16) : "memory");
      turn_of<kAhead>(fn, g, from);
    }
    const int left = whole - first - turns * kTurn;
    if (left >= 2 * kTeam) turn_of<2>(fn, g, from);
    const int end = past + (with_head ? head : 0);
    if (g >= end) return;
    Group<T> next = masked(g == past ? 0 : g);
#pragma unroll 1
    do {
      Group<T> v[1] = {next};
      const int at = g == past ? 0 : g;
      g += kTeam;
      if (g < end) next = masked(g == past ? 0 : g);
      fn(v, at);
    } while (g < end);
  }
  template <typename Fn>
  __device__ __forceinline__ void each(Fn& fn) const { each(fn, head, groups, true); }

  // The lanes of the thread's team within its warp. The teams of a warp part where one row takes a branch and another does not
  // (an infinity, a temperature of 0), so what they do together names no lane of another team.
  __device__ __forceinline__ static uint32_t mates() {
    return kTeam < 32 ? ((1u << (kTeam & 31)) - 1) << (threadIdx.x & 31 & -kTeam) : 0xffffffffu;
  }
  __device__ __forceinline__ void team_sync() const {
    if (kTeam <= 32) __syncwarp(mates());
    else __syncthreads();
  }
  __device__ void row_sync() {
    if (blocks > 1) cluster.sync();
    else team_sync();
  }
  // One barrier for each of these: what a warp finds is combined by every warp again.
  __device__ uint32_t team_max(uint32_t v) {
    if (kTeam < 32) {
#pragma unroll
      for (int o = kTeam / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(mates(), v, o));
      return v;
    }
    v = __reduce_max_sync(0xffffffffu, v);
    if (kTeam == 32) return v;
    uint32_t* const part = reinterpret_cast<uint32_t*>(scratch + 32 * (turn ^= 1));
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < kWarps ? part[lane] : 0);
  }
  __device__ __forceinline__ static float more(float v, int o) { return v + __shfl_xor_sync(mates(), v, o); }
  __device__ __forceinline__ static void more(float2& v, int o) { v.x = more(v.x, o), v.y = more(v.y, o); }
  __device__ __forceinline__ static void more(float3& v, int o) { v.x = more(v.x, o), v.y = more(v.y, o), v.z = more(v.z, o); }
  template <typename V>
  __device__ static V warp_sum(V v) {
#pragma unroll
    for (int o = kTeam < 32 ? kTeam / 2 : 16; o; o >>= 1) more(v, o);
    return v;
  }
  // Two or three sums.
  template <typename V>
  __device__ V team_sum(V v) {
    v = warp_sum(v);
    if (kTeam <= 32) return v;
    V* const part = reinterpret_cast<V*>(scratch + 32 * (turn ^= 1));
    if (lane == 0) part[warp] = v;
    __syncthreads();
    return warp_sum(lane < kWarps ? part[lane] : V{});
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
  // The largest of a group's scores; NaN is passed over.
  __device__ __forceinline__ static float largest(const Group<T>& v) {
    if constexpr (kG == 4) {
      return fmaxf(fmaxf(v.get(0), v.get(1)), fmaxf(v.get(2), v.get(3)));
    } else {
      typedef std::conditional_t<std::is_same<T, __half>::value, __half2, __nv_bfloat162> T2;
      const T2* const p = reinterpret_cast<const T2*>(&v.u);
      const T2 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
      return fmaxf(float(m.x), float(m.y));
    }
  }
  // Some entries. kMean: also the sum of w d.
  template <bool kMean, int kN>
  __device__ __forceinline__ void add(const Group<T> (&v)[kN]) {
    float most = largest(v[0]);
#pragma unroll
    for (int u = 1; u < kN; u++) most = fmaxf(most, largest(v[u]));
    if (most > own.m) {
      shift(own, most, per);
      s_low = e_low = 0.f;
    }
    if (own.m == -INFINITY) return;
    float2 w = make_float2(0.f, 0.f), e = w;
#pragma unroll
    for (int u = 0; u < kN; u++) {
      float s[kG];
      floats(v[u], s);
#pragma unroll
      for (int j = 0; j < kG; j += 2) {
        const float2 d = far2(s[j], s[j + 1], own.m, per), x = make_float2(fast_exp2(d.x), fast_exp2(d.y));
        w = add2(w, x);
        if (kMean) e = fma2(d, x, e);
      }
    }
    add_kept(own.s, s_low, w.x + w.y);
    if (kMean) add_kept(own.e, e_low, e.x + e.y);
  }
  struct Add {
    Row& r;
    template <int kN>
    __device__ __forceinline__ void operator()(const Group<T> (&v)[kN], int) { r.template add<true>(v); }
  };
  // Of all entries.
  __device__ __forceinline__ void sum_up() {
    begin();
    Add add_all{*this};
    each(add_all);
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
    for (int g = tid; g < groups; g += kTeam) {
      const Group<T> v = masked(g);
#pragma unroll
      for (int j = 0; j < kG; j++)
        if (v.get(j) == m) from_end = max(from_end, 0xffffffffu - uint32_t(lo + g * kG - skip + j));
    }
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
  __device__ __forceinline__ static void pair_as(float* d, float x, float y) { d[0] = x, d[1] = y; }
  __device__ __forceinline__ static void pair_as(__nv_bfloat16* d, float x, float y) { *reinterpret_cast<__nv_bfloat162*>(d) = __floats2bfloat162_rn(x, y); }
  __device__ __forceinline__ static void pair_as(__half* d, float x, float y) { *reinterpret_cast<__half2*>(d) = __floats2half2_rn(x, y); }
  template <typename D>
  __device__ __forceinline__ static void store_whole(uint8_t* p, const float (&v)[kG]) {
    constexpr int kBytes = kG * int(sizeof(D));
    uint32_t w[kBytes / 4];
    D* const d = reinterpret_cast<D*>(w);
#pragma unroll
    for (int j = 0; j < kG; j += 2) pair_as(d + j, v[j], v[j + 1]);
    if (kBytes == 8) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
#pragma unroll
    for (int k = 0; k < kBytes / 16; k++)
      __stcs(reinterpret_cast<uint4*>(p) + k, make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]));
  }
  // What f makes of the groups' scores (two at a time) to their places in the gradient.
  template <int kN, typename F>
  __device__ __forceinline__ void store(const Out& o, const Group<T> (&v)[kN], int g, F& f) const {
    const int i = g * kG - skip;
    uint8_t* const p = o.p + int64_t(i) * o.size;
    if (o.whole && (kN > 1 || (i >= 0 && i + kG <= count))) {
      if (o.dtype == EMR_F32) store_as<float>(p, v, f);
      else if (o.dtype == EMR_BF16) store_as<__nv_bfloat16>(p, v, f);
      else store_as<__half>(p, v, f);
    } else {
#pragma unroll
      for (int u = 0; u < kN; u++) {
        float s[kG];
        made(v[u], s, f);
#pragma unroll
        for (int j = 0; j < kG; j++) {
          const int at = i + u * kTeam * kG + j;
          if (kN > 1 || unsigned(at) < unsigned(count)) store_scalar(o.p, o.dtype, at, s[j]);
        }
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ static void made(const Group<T>& v, float (&s)[kG], F& f) {
    floats(v, s);
#pragma unroll
    for (int j = 0; j < kG; j += 2) {
      const float2 y = f(s[j], s[j + 1]);
      s[j] = y.x, s[j + 1] = y.y;
    }
  }
  template <typename D, int kN, typename F>
  __device__ __forceinline__ static void store_as(uint8_t* p, const Group<T> (&v)[kN], F& f) {
#pragma unroll
    for (int u = 0; u < kN; u++) {
      float s[kG];
      made(v[u], s, f);
      store_whole<D>(p + u * kTeam * kG * int(sizeof(D)), s);
    }
  }
  // The whole slice.
  template <typename F>
  struct Put {
    const Row& r;
    const Out& o;
    F& f;
    template <int kN>
    __device__ __forceinline__ void operator()(const Group<T> (&v)[kN], int g) { r.store(o, v, g, f); }
  };
  template <typename F>
  __device__ __forceinline__ void put(const Out& o, F f) const {
    Put<F> all{*this, o, f};
    each(all);
  }
};

template <typename A>
emr_status launch_rows(void (*kernel)(A), const A& a, int team, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  const int rows = team <= 32 ? 256 / team : 1;  // of a block
  cfg.gridDim = dim3(unsigned((int64_t(a.rows) + rows - 1) / rows) * unsigned(cluster));
  cfg.blockDim = dim3(unsigned(team * rows));
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
    else cudaGetLastError();  // the question's error is not the caller's
  }
}

// Smaller teams where rows are many and short: what a row costs beside its entries, about 250 instructions a warp for the
// sums, 500 in a gradient and 750 in distillation, counts for each of its warps, and more rows are at hand while one waits.
// Gradients of bfloat16 by 64 and by 128 threads: 2000 x 5460 13.7 and 17.4 us, 8000 x 1364 23 and 34; best 20 of float32
// 2000 x 1364 10.1 and 11.3, 1000 x 1364 8.2 and 7.3, 4000 x 5460 38 and 33.
// The other steps, in us on the device with 152 SMs, the rule's choice first where nothing else is said.
// 8 threads or 32, gradients: 4864 x 340 bfloat16 6.2 and 7.5, 9728 x 512 6.5 and 9.0, 4864 x 512 float32 5.8 and 5.2; below, 32 or 8: 2432 x 340
// 5.2 and 6.2, 4864 x 1024 7.2 and 7.2, but 9728 x 700 13.6 and 9.2.
// 32 threads or 64, bfloat16: gradients of 2432 x 340 5.2 and 6.8, of 2432 x 1024 4.8 and 5.9; best 5 of 2432 x 1024 5.5 and 7.5, best 20 9.9 and 9.2,
// but best 32 37.9 and 11.3; distillation with lists of 16 9.1 and 11.3, of 64 18.8 and 16.4. Below, 64 or 32: gradients of 1216 x 340 4.8 and 4.8, of
// 1216 x 700 5.5 and 4.8.
// 128 threads or 256: sums of 608 x 5460 bfloat16 4.8 and 4.5, gradients of 608 x 8192 6.5 and 6.9, best 20 8.6 and 8.8; 256 or 128: gradients of
// 304 x 5460 float32 5.2 and 5.5.
// 256 threads or a block of 512, float32: sums of 152 x 8192 3.4 and 3.8, gradients 4.1 and 4.5, best 20 7.2 and 7.5. A row of more than 8,192 that gets
// one block, 512 or 256: gradients of 608 x 40000 39.5 and 47.5, but of 608 x 12000 17.6 and 14.4, best 20 of 608 x 20001 26.3 and 19.9.
// Clusters of 1, 2, 4 and 8, gradients of float32: 20 x 40000 8.9, 7.9, 6.2 and 7.2 (taken: 8), 64 x 40000 8.9, 7.9, 8.1 and 13.9 (4), 152 x 40000 14.1, 14.5, 22.8
// and 34.4 (2), 1 x 20001 6.4, 5.8, 5.8 and 6.2 (4); 152 x 12000 5.5, 7.2, 15.4 and 24.9 (2, as best 20, 8.6 and 13.7 of one and two): entries of a block, 4,096
// at least, could be twice as many.
// The team and cluster of a row, and the slice of its blocks: the same with and without a gradient, so that the values are.
// least: the smallest team that will do; size: bytes of a score.
inline int plan(Rows& a, int least, int size, int sms, const int* fit, int* cluster) {
  *cluster = 1;
  a.slice = (a.n + 15) / 16 * 16;
  if (a.n <= 8192) {
    if (least <= 8 && a.n <= 512 && a.rows >= 32 * sms) return 8;
    if (least <= 32 && a.n <= 1024 && a.rows >= 16 * sms) return 32;
    if (least <= 64 && a.n * size <= 12288 && a.rows >= 8 * sms) return 64;
    return least <= 128 && a.rows >= 4 * sms ? 128 : 256;
  }
  for (int c = 2; c <= kMaxCluster; c++)
    if (a.rows <= fit[c] && a.n / c >= 4096) *cluster = c;
  // a row that is read again, for its gradient, should still be in L2
  while (2 * *cluster <= kMaxCluster && a.n / (2 * *cluster) >= 8192 && 2. * sms / *cluster * double(a.n) * size > double(64 << 20)) *cluster *= 2;
  a.slice = ((a.n + *cluster - 1) / *cluster + 15) / 16 * 16;
  return 512;
}

inline bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline emr_status check_scores(const void* scores, int32_t dtype, int32_t rows, int64_t n, int64_t row_stride) {
  if (rows < 1 || n < 1 || !scores || !dtype_ok(dtype) || row_stride < 0 || !aligned(scores, dtype_bytes(dtype))) return EMR_ERR_ARG;
  return n > (int64_t(1) << 31) - (1 << 20) || rows > (1 << 27) ? EMR_ERR_RANGE : EMR_OK;
}

}  // namespace rows
}  // namespace emr
